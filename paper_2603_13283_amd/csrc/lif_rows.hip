// lif_rows.hip -- probabilities read off rows of logits: log probabilities of
// given tokens with entropy and the likeliest alternatives
// (lif_token_logprobs), and distillation from a teacher's likeliest classes
// (lif_distill_top), each with its gradient.
//
// With m the row's largest logit and c = log2(e) / temperature, every term
// is e_j = 2^{(x_j - m) c}; S = sum e_j gives p_j = e_j / S and
// lse = m / temperature + log S.
#include "lif_host.hpp"
#include "lif_types.hpp"

namespace lif {
namespace {

constexpr int kRowThreads = 256;
constexpr float kLn2 = 0.693147180559945309f;
constexpr float kNegInf = -INFINITY;

struct RowArgs {
    int R, V, k;
    int64_t stride, grad_stride;
    float c, inv_t;             // log2(e) / temperature, 1 / temperature
    double inv_td;
    bool tail;
};

// Orders float32 values as unsigned integers; -0 and +0 are equal, a NaN
// ranks below -infinity.
__device__ __forceinline__ uint32_t order_key(float v)
{
    if (v != v) return 0;
    const uint32_t u = __float_as_uint(v + 0.0f);
    return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

__device__ __forceinline__ float wave_sum(float v)
{
    for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
    return v;
}
__device__ __forceinline__ float wave_max(float v)
{
    for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
    return v;
}

struct Shared {
    float part[4][kRowThreads / 64];
    unsigned long long best[kRowThreads / 64];
};

__device__ __forceinline__ float block_sum(float v, float* part)
{
    v = wave_sum(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = 0.0f;
    for (int i = 0; i < kRowThreads / 64; ++i) s += part[i];
    return s;
}
__device__ __forceinline__ float block_max(float v, float* part)
{
    v = wave_max(v);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    float s = part[0];
    for (int i = 1; i < kRowThreads / 64; ++i) s = fmaxf(s, part[i]);
    return s;
}

// (x - m) c; 0 for the row's largest logits, also where they are infinite
// or the row has nothing above -infinity.
__device__ __forceinline__ float log2_term(float x, float m, float c) { return (x - m) * c; }

template <typename E>
__global__ __launch_bounds__(kRowThreads) void k_token_logprobs(
    const E* __restrict__ logits, const int32_t* __restrict__ token, RowArgs a, float* __restrict__ logp,
    float* __restrict__ entropy, float* __restrict__ lse, float* __restrict__ top_logp, int32_t* __restrict__ top_idx,
    const float* __restrict__ g_logp, const float* __restrict__ g_ent, E* __restrict__ grad)
{
    __shared__ Shared sh;
    const int r = blockIdx.x, tid = threadIdx.x;
    const E* x = logits + r * a.stride;
    float m = kNegInf;
    for (int j = tid; j < a.V; j += kRowThreads) m = fmaxf(m, to_f32(x[j]));
    m = block_max(m, sh.part[0]);
    const float ms = m == kNegInf ? 0.0f : m;
    float s = 0.0f, u = 0.0f;
    for (int j = tid; j < a.V; j += kRowThreads) {
        const float z = log2_term(to_f32(x[j]), ms, a.c), e = exp2f(z);
        s += e;
        u = fmaf(e, fmaxf(z, -200.0f), u);
    }
    s = block_sum(s, sh.part[0]);
    u = block_sum(u, sh.part[1]);
    const bool empty = s == 0.0f;
    const float ls = empty ? kNegInf : logf(s);
    const float H = empty ? 0.0f : ls - kLn2 * (u / s);
    const int tok = token ? token[r] : -1;
    const bool there = tok >= 0 && tok < a.V;
    if (tid == 0) {
        if (logp) logp[r] = !there ? 0.0f : empty ? kNegInf : (to_f32(x[tok]) - ms) * a.inv_t - ls;
        if (entropy) entropy[r] = H;
        if (lse) lse[r] = empty ? kNegInf : (float)((double)ms * a.inv_td + (double)ls);
    }
    unsigned long long last = ~0ull;
    for (int i = 0; i < a.k; ++i) {          // the largest key below the last one
        unsigned long long best = 0;
        for (int j = tid; j < a.V; j += kRowThreads) {
            const unsigned long long key = ((unsigned long long)order_key(to_f32(x[j])) << 32) | (0xffffffffu - (uint32_t)j);
            if (key < last && key > best) best = key;
        }
        for (int o = 32; o; o >>= 1) {
            const unsigned long long w = __shfl_xor(best, o);
            best = w > best ? w : best;
        }
        __syncthreads();
        if ((tid & 63) == 0) sh.best[tid >> 6] = best;
        __syncthreads();
        for (int q = 0; q < kRowThreads / 64; ++q) best = sh.best[q] > best ? sh.best[q] : best;
        last = best;
        if (tid == 0) {
            const int j = (int)(0xffffffffu - (uint32_t)best);
            top_idx[(int64_t)r * a.k + i] = j;
            top_logp[(int64_t)r * a.k + i] = empty ? kNegInf : (to_f32(x[j]) - ms) * a.inv_t - ls;
        }
    }
    if (!grad) return;
    const float g = there && g_logp ? g_logp[r] : 0.0f, ge = g_ent ? g_ent[r] : 0.0f;
    const float inv_s = empty ? 0.0f : 1.0f / s;
    for (int j = tid; j < a.V; j += kRowThreads) {
        const float z = log2_term(to_f32(x[j]), ms, a.c);
        const float p = exp2f(z) * inv_s;
        const float lp = empty ? 0.0f : fmaf(kLn2, fmaxf(z, -200.0f), -ls);
        float v = -p * fmaf(ge, lp + H, g);
        if (there && j == tok && !empty) v += g;
        grad[r * a.grad_stride + j] = from_f32<E>(v * a.inv_t);
    }
}

template <typename E>
__global__ __launch_bounds__(kRowThreads) void k_distill(const E* __restrict__ logits,
                                                         const float* __restrict__ t_logp,
                                                         const int32_t* __restrict__ t_idx, RowArgs a,
                                                         const float* __restrict__ weight, float* __restrict__ loss,
                                                         E* __restrict__ grad)
{
    __shared__ Shared sh;
    __shared__ int li[LIF_TOP_MAX];
    __shared__ float lq[LIF_TOP_MAX], lt[LIF_TOP_MAX];
    const int r = blockIdx.x, tid = threadIdx.x;
    const E* x = logits + r * a.stride;
    if (tid < a.k) {
        const int j = t_idx[(int64_t)r * a.k + tid];
        const bool used = j >= 0 && j < a.V;
        li[tid] = used ? j : -1;
        lt[tid] = used ? t_logp[(int64_t)r * a.k + tid] : kNegInf;
        lq[tid] = used ? expf(lt[tid]) : 0.0f;
    }
    float m = kNegInf;
    for (int j = tid; j < a.V; j += kRowThreads) m = fmaxf(m, to_f32(x[j]));
    m = block_max(m, sh.part[0]);
    const float ms = m == kNegInf ? 0.0f : m;
    double sq = 0.0;
    for (int i = 0; i < a.k; ++i) sq += (double)lq[i];
    float s_top = 0.0f, s_rest = 0.0f;
    int n_top = 0;
    for (int j = tid; j < a.V; j += kRowThreads) {
        const float e = exp2f(log2_term(to_f32(x[j]), ms, a.c));
        bool in = false;
        for (int i = 0; i < a.k; ++i) in |= li[i] == j;
        if (in) { s_top += e; ++n_top; } else s_rest += e;
    }
    s_top = block_sum(s_top, sh.part[0]);
    s_rest = block_sum(s_rest, sh.part[1]);
    const float n_in = block_sum((float)n_top, sh.part[2]);
    const float s = s_top + s_rest;
    const bool empty = s == 0.0f, none = sq == 0.0;
    const float ls = empty ? kNegInf : logf(s);
    double q_rest = 0.0;
    if (a.tail && 1.0 - sq >= LIF_DISTILL_TAIL_MIN && n_in < (float)a.V) q_rest = 1.0 - sq;
    const double scale = a.tail ? 1.0 : 1.0 / sq;
    if (tid == 0 && loss) {
        double v = 0.0;
        for (int i = 0; i < a.k && !none; ++i) {
            const double q = (double)lq[i] * scale;
            if (q > 0.0) {
                const double lp = empty ? (double)kNegInf
                                        : ((double)to_f32(x[li[i]]) - (double)ms) * a.inv_td - (double)ls;
                v += q * ((double)lt[i] + log(scale) - lp);
            } else if (q != q) v = q;
        }
        if (!none && q_rest > 0.0) v += q_rest * (log(q_rest) - (empty ? (double)kNegInf : log((double)s_rest) - log((double)s)));
        loss[r] = (float)v;
    }
    if (!grad) return;
    const float w = (weight ? weight[r] : 1.0f) * a.inv_t;
    const double mass = a.tail ? sq + q_rest : 1.0;
    const float c_top = none || empty ? 0.0f : (float)(mass / (double)s);
    const float c_rest = none || empty ? 0.0f : q_rest > 0.0 && s_rest > 0.0f ? (float)(mass / (double)s - q_rest / (double)s_rest) : c_top;
    for (int j = tid; j < a.V; j += kRowThreads) {
        const float e = exp2f(log2_term(to_f32(x[j]), ms, a.c));
        double q = 0.0;
        bool in = false;
        for (int i = 0; i < a.k; ++i)
            if (li[i] == j) { in = true; q += (double)lq[i] * scale; }
        const float v = none || empty ? 0.0f : in ? fmaf(e, c_top, -(float)q) : e * c_rest;
        grad[r * a.grad_stride + j] = from_f32<E>(v * w);
    }
}

int check_rows(const lif_rows_params* p)
{
    if (!p || p->R < 0 || p->V < 1 || p->k < 0 || p->k > p->V || p->reserved != 0) return LIF_ERR_ARG;
    if (p->dtype != LIF_F32 && p->dtype != LIF_BF16 && p->dtype != LIF_F16) return LIF_ERR_ARG;
    if (p->flags & ~LIF_DISTILL_TAIL) return LIF_ERR_ARG;
    if (p->stride < p->V || p->grad_stride < p->V) return LIF_ERR_ARG;
    if (!(p->temperature >= 1.0 / 1048576.0 && p->temperature <= 1048576.0)) return LIF_ERR_ARG;
    if (p->k > LIF_TOP_MAX) return LIF_ERR_SIZE;
    return LIF_OK;
}

RowArgs row_args(const lif_rows_params& p)
{
    RowArgs a;
    a.R = p.R;
    a.V = p.V;
    a.k = p.k;
    a.stride = p.stride;
    a.grad_stride = p.grad_stride;
    a.c = (float)(1.4426950408889634074 / p.temperature);
    a.inv_t = (float)(1.0 / p.temperature);
    a.inv_td = 1.0 / p.temperature;
    a.tail = p.flags & LIF_DISTILL_TAIL;
    return a;
}

}  // namespace
}  // namespace lif

extern "C" size_t lif_rows_workspace_size(const lif_rows_params* p)
{
    if (lif::check_rows(p) != LIF_OK) return 0;
    return 0;
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
    const size_t need = lif_rows_workspace_size(p);
    if (need > 0 && !ws) return LIF_ERR_ARG;
    if (ws_bytes < need) return LIF_ERR_WORKSPACE;
    if (p->R == 0) return LIF_OK;
    RowArgs a = row_args(*p);
    if (!top_idx) a.k = 0;
    with_dtype(p->dtype, [&](auto tag) {
        using E = decltype(tag);
        TIMED_LAUNCH("token_logprobs", k_token_logprobs<E>, dim3(p->R), dim3(kRowThreads), 0, (hipStream_t)stream,
                     (const E*)logits, token, a, logp, entropy, lse, top_logp, top_idx, grad_logp, grad_entropy,
                     (E*)grad);
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
    const size_t need = lif_rows_workspace_size(p);
    if (need > 0 && !ws) return LIF_ERR_ARG;
    if (ws_bytes < need) return LIF_ERR_WORKSPACE;
    if (p->R == 0) return LIF_OK;
    const RowArgs a = row_args(*p);
    with_dtype(p->dtype, [&](auto tag) {
        using E = decltype(tag);
        TIMED_LAUNCH("distill_top", k_distill<E>, dim3(p->R), dim3(kRowThreads), 0, (hipStream_t)stream,
                     (const E*)logits, teacher_logp, teacher_idx, a, weight, loss, (E*)grad);
    });
    return check_launch();
}
