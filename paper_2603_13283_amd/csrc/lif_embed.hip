// lif_embed.hip -- rows of a table by token (lif_embed), and the gradient of
// the table (lif_embed_backward).
//
// The gradient sorts the places of the tokens, stably and by counting: a digit
// at a time, each of up to 256 workgroups counts the digits of its chunk of
// places, the counts are summed over chunks, and every workgroup hands out the
// places of its chunk in order.  Then each row of the table has its places in
// one run; the list is cut into pieces of equal length that waves sum up, and
// runs that cross pieces are joined in the order of the pieces.  The order of
// all sums follows from tokens and sizes alone.
#include "lif_host.hpp"
#include "lif_types.hpp"
#include "lif_walk.hpp"

namespace lif {
namespace {

constexpr int kMaxBits = 10;          // of a digit
constexpr int kChunks = 256;          // workgroups that count and hand out
constexpr int kSortWaves = 4;
constexpr int kFew = 4096, kSmallWaves = 16;      // places that one workgroup sorts
constexpr int kAhead = 8;             // rows whose loads are in flight at once
constexpr int kJoinWaves = 8;
constexpr int kSeek = 16;             // lanes that look for a row of the table together

// The row of place i, V where it has none.
__device__ __forceinline__ uint32_t key_of(const int32_t* __restrict__ token, const int32_t* __restrict__ length,
                                           int T, int V, int i)
{
    const int v = token[i];
    bool on = v >= 0 && v < V;
    if (length && on) {
        const int b = i / T;
        on = i - b * T < length[b];
    }
    return on ? (uint32_t)v : (uint32_t)V;
}

// Vectors of VEC elements; where VEC does not divide D, a row's last one starts
// at D - VEC and repeats some of the one before.  Bound by writes: 160000 x 256
// f32 28 us, 164 MB at 5.8 TB/s; the table comes from the caches.
template <typename E, typename F, int VEC>
__global__ __launch_bounds__(256) void k_embed(const int32_t* __restrict__ token, const E* __restrict__ W,
                                               const int32_t* __restrict__ length, int T, int V, int D, int groups,
                                               int rows, int64_t w_row, float scale, int R, F* __restrict__ out)
{
    const int64_t r0 = (int64_t)blockIdx.x * rows, items = (int64_t)min((int64_t)rows, R - r0) * groups;
    for (int64_t j = threadIdx.x; j < items; j += 256) {
        const int64_t r = r0 + j / groups;
        const int d = min((int)(j % groups) * VEC, D - VEC);
        const uint32_t v = key_of(token, length, T, V, (int)r);
        E e[VEC];
        F o[VEC];
        if (v < (uint32_t)V) load_elems<E, VEC>(W + (int64_t)v * w_row + d, e);
#pragma unroll
        for (int k = 0; k < VEC; ++k) o[k] = from_f32<F>(v < (uint32_t)V ? to_f32(e[k]) * scale : 0.0f);
        store_elems<F, VEC>(out + r * D + d, o);
    }
}

struct Sort {
    int R, T, V, chunk, bits, shift;
};

// Counts of a chunk's digits.
__global__ __launch_bounds__(kSortWaves* kWave) void k_count(const int32_t* __restrict__ token,
                                                             const int32_t* __restrict__ length,
                                                             const uint32_t* __restrict__ keys, Sort q,
                                                             uint32_t* __restrict__ count)
{
    __shared__ uint32_t sh[1 << kMaxBits];
    const int bins = 1 << q.bits, c = blockIdx.x;
    for (int i = threadIdx.x; i < bins; i += kSortWaves * kWave) sh[i] = 0;
    __syncthreads();
    const int64_t end = min((int64_t)(c + 1) * q.chunk, (int64_t)q.R);
    for (int64_t i = (int64_t)c * q.chunk + threadIdx.x; i < end; i += kSortWaves * kWave) {
        const uint32_t k = keys ? keys[i] : key_of(token, length, q.T, q.V, (int)i);
        atomicAdd(&sh[(k >> q.shift) & (bins - 1)], 1u);
    }
    __syncthreads();
    for (int i = threadIdx.x; i < bins; i += kSortWaves * kWave) count[(int64_t)c * bins + i] = sh[i];
}

// Per digit: the counts become sums over the chunks before, total the whole.
// A workgroup takes 64 digits, its 16 waves 16 chunks each, all their loads in
// flight at once (one wave over all chunks: 30 us, this 3).
__global__ __launch_bounds__(16 * kWave) void k_chunk_sums(uint32_t* __restrict__ count, int chunks, int bins,
                                                           uint32_t* __restrict__ total)
{
    constexpr int kEach = kChunks / 16;
    __shared__ uint32_t sh[16][kWave];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, d = blockIdx.x * kWave + lane;
    uint32_t v[kEach], s = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int c = w * kEach + i;
        v[i] = d < bins && c < chunks ? count[(int64_t)c * bins + d] : 0;
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) s += v[i];
    sh[w][lane] = s;
    __syncthreads();
    uint32_t before = 0, all = 0;
    for (int i = 0; i < 16; ++i) {
        before += i < w ? sh[i][lane] : 0;
        all += sh[i][lane];
    }
    if (d >= bins) return;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
        const int c = w * kEach + i;
        if (c < chunks) count[(int64_t)c * bins + d] = before;
        before += v[i];
    }
    if (w == 0) total[d] = all;
}

// Hands out a chunk's places in order.  Each wave takes a contiguous part of
// the chunk, 64 places at a time: lanes of the same digit find each other by
// ballots over its bits.
__global__ __launch_bounds__(kSortWaves* kWave) void k_hand_out(const int32_t* __restrict__ token,
                                                                const int32_t* __restrict__ length,
                                                                const uint32_t* __restrict__ keys,
                                                                const uint32_t* __restrict__ places, Sort q,
                                                                const uint32_t* __restrict__ count,
                                                                const uint32_t* __restrict__ total,
                                                                uint32_t* __restrict__ keys_out,
                                                                uint32_t* __restrict__ places_out,
                                                                uint32_t* __restrict__ list)
{
    if (blockIdx.x == 0 && threadIdx.x == 0) *list = 0;
    constexpr int kThreads = kSortWaves * kWave, kPer = (1 << kMaxBits) / kThreads;
    __shared__ uint32_t next[kSortWaves][1 << kMaxBits], waves[kSortWaves];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6, bins = 1 << q.bits, c = blockIdx.x;
    for (int i = threadIdx.x; i < bins; i += kThreads)
        for (int j = 0; j < kSortWaves; ++j) next[j][i] = 0;
    // where each digit begins: a scan of the totals, kPer adjacent ones a thread
    uint32_t mine[kPer], sum = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int d = threadIdx.x * kPer + i;
        mine[i] = d < bins ? total[d] : 0;
        sum += mine[i];
    }
    uint32_t before = sum;
    for (int o = 1; o < kWave; o <<= 1) {
        const uint32_t v = __shfl_up(before, o);
        if (lane >= o) before += v;
    }
    if (lane == kWave - 1) waves[w] = before;
    __syncthreads();
    before -= sum;
    for (int i = 0; i < w; ++i) before += waves[i];
    // the waves' counts, then where each wave's places of a digit begin
    const int64_t first = (int64_t)c * q.chunk;
    const int n = (int)min((int64_t)q.chunk, (int64_t)q.R - first), part = q.chunk / kSortWaves;
    const int from = min(w * part, n), end = min(from + part, n);
    auto key_at = [&](int64_t i) { return keys ? keys[i] : key_of(token, length, q.T, q.V, (int)i); };
    for (int i = from + lane; i < end; i += kWave)
        atomicAdd(&next[w][(key_at(first + i) >> q.shift) & (bins - 1)], 1u);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const int d = threadIdx.x * kPer + i;
        if (d < bins) {
            uint32_t at = before + count[(int64_t)c * bins + d];
            for (int j = 0; j < kSortWaves; ++j) {
                const uint32_t v = next[j][d];
                next[j][d] = at;
                at += v;
            }
            before += mine[i];
        }
    }
    __syncthreads();
    for (int i0 = 0; i0 < part; i0 += kWave) {
        const bool on = from + i0 + lane < end;
        const int64_t i = first + (on ? from + i0 + lane : 0);
        const uint32_t k = key_at(i);
        const uint32_t digit = (k >> q.shift) & (bins - 1);
        uint64_t same = __ballot(on);
        for (int b = 0; b < q.bits; ++b) {
            const uint64_t set = __ballot((digit >> b) & 1);
            same &= (digit >> b) & 1 ? set : ~set;
        }
        const int rank = __popcll(same & (((uint64_t)1 << lane) - 1));
        uint32_t at = 0;
        if (on) at = next[w][digit] + rank;
        __syncthreads();
        if (on && rank == 0) next[w][digit] = at + __popcll(same);
        __syncthreads();
        if (on) {
            keys_out[at] = k;
            places_out[at] = places ? places[i] : (uint32_t)i;
        }
    }
}

// Few places: one workgroup sorts them in LDS, 8 bits of the key at a time, in
// the same way (1000 places, 200 rows of the table 23.5 -> 17.7 us a call, 50000 rows
// 31.7 -> 18.5; at 8000 places no gain).
__global__ __launch_bounds__(kSmallWaves* kWave) void k_sort_few(const int32_t* __restrict__ token,
                                                                 const int32_t* __restrict__ length, Sort q,
                                                                 uint32_t* __restrict__ keys_out,
                                                                 uint32_t* __restrict__ places_out,
                                                                 uint32_t* __restrict__ list)
{
    if (threadIdx.x == 0) *list = 0;
    constexpr int kThreads = kSmallWaves * kWave, kBins = 256;
    __shared__ uint32_t key[2][kFew], next[kSmallWaves][kBins], waves[kBins / kWave];
    __shared__ uint16_t place[2][kFew];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    for (int i = threadIdx.x; i < q.R; i += kThreads) {
        key[0][i] = key_of(token, length, q.T, q.V, i);
        place[0][i] = (uint16_t)i;
    }
    const int part = (q.R + kThreads - 1) / kThreads * kWave, from = min(w * part, q.R), end = min(from + part, q.R);
    int now = 0;
    for (int shift = 0; shift < q.bits; shift += 8, now ^= 1) {
        for (int i = threadIdx.x; i < kSmallWaves * kBins; i += kThreads) (&next[0][0])[i] = 0;
        __syncthreads();
        for (int i = from + lane; i < end; i += kWave) atomicAdd(&next[w][(key[now][i] >> shift) & (kBins - 1)], 1u);
        __syncthreads();
        uint32_t count = 0, before = 0;
        if (threadIdx.x < kBins) {
            for (int j = 0; j < kSmallWaves; ++j) count += next[j][threadIdx.x];
            before = count;
            for (int o = 1; o < kWave; o <<= 1) {
                const uint32_t v = __shfl_up(before, o);
                if (lane >= o) before += v;
            }
            if (lane == kWave - 1) waves[w] = before;
        }
        __syncthreads();
        if (threadIdx.x < kBins) {
            before -= count;
            for (int j = 0; j < w; ++j) before += waves[j];
            for (int j = 0; j < kSmallWaves; ++j) {
                const uint32_t v = next[j][threadIdx.x];
                next[j][threadIdx.x] = before;
                before += v;
            }
        }
        __syncthreads();
        const bool last = shift + 8 >= q.bits;
        for (int i0 = 0; i0 < part; i0 += kWave) {
            const bool on = from + i0 + lane < end;
            const int i = on ? from + i0 + lane : 0;
            const uint32_t k = key[now][i], digit = (k >> shift) & (kBins - 1);
            uint64_t same = __ballot(on);
            for (int b = 0; b < 8; ++b) {
                const uint64_t set = __ballot((digit >> b) & 1);
                same &= (digit >> b) & 1 ? set : ~set;
            }
            const int rank = __popcll(same & (((uint64_t)1 << lane) - 1));
            uint32_t at = 0;
            if (on) at = next[w][digit] + rank;
            __syncthreads();
            if (on && rank == 0) next[w][digit] = at + __popcll(same);
            __syncthreads();
            if (on && last) keys_out[at] = k, places_out[at] = place[now][i];
            if (on && !last) key[now ^ 1][at] = k, place[now ^ 1][at] = place[now][i];
        }
        __syncthreads();
    }
}

struct Sums {
    int R, T, V, D, piece, pieces, columns;
    int64_t g_batch, g_time;
    float scale;
};

__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __builtin_amdgcn_readfirstlane(v); }

// Whether row v of the table is named, looked for by kSeek lanes at once: each
// step leaves one of kSeek + 1 parts of the list.
__device__ __forceinline__ bool named(const uint32_t* __restrict__ keys, int R, uint32_t v, int lane)
{
    int lo = 0, hi = R;                                             // the first key of at least v is in [lo, hi]
    const int sub = lane & (kSeek - 1), shift = lane & ~(kSeek - 1);
    while (__any(lo < hi)) {
        const int at = lo + (int)((int64_t)(hi - lo) * (sub + 1) / (kSeek + 1));
        const bool less = lo < hi && keys[at] < v;
        const int below = __popcll((__ballot(less) >> shift) & ((1u << kSeek) - 1));
        const int from = __shfl(at, shift + max(below - 1, 0)), to = __shfl(at, shift + min(below, kSeek - 1));
        if (lo < hi) {
            const int l = below > 0 ? from + 1 : lo;
            hi = below < kSeek ? to : hi;
            lo = l;
        }
    }
    return lo < R && keys[lo] == v;
}

// A wave sums the rows of a piece of the sorted list for 64 VEC columns.  A run
// that lies within the piece goes to the table's gradient, one that comes from
// the piece before to part[piece][0], one that begins here and goes on to
// part[piece][1], and the piece to the list of those whose run is joined later
// (list[0] counts them; their order there is open, and without effect).  The
// workgroups from sum_blocks on clear the rows that no token names.  Bound by memory:
// 32768 x 1001 bf16 into 50021 rows 46 us, 266 MB at 5.8 TB/s; half of 160000 x 256
// f32 into 700 rows 19 us, 82 MB at 4.3 TB/s.
template <typename E, int VEC>
__global__ __launch_bounds__(256) void k_embed_sums(const E* __restrict__ grad, const uint32_t* __restrict__ keys,
                                                    const uint32_t* __restrict__ places, Sums q, int64_t sum_blocks,
                                                    float* __restrict__ gW, float* __restrict__ part,
                                                    uint32_t* __restrict__ list)
{
    const int lane = threadIdx.x & 63;
    if (blockIdx.x >= sum_blocks) {
        const int64_t v0 = ((blockIdx.x - sum_blocks) * 4 + (threadIdx.x >> 6)) * (kWave / kSeek);
        const int64_t v = v0 + lane / kSeek;
        const bool missing = !named(keys, q.R, (uint32_t)min(v, (int64_t)q.V - 1), lane) && v < q.V;
        uint64_t rows = __ballot(missing && (lane & (kSeek - 1)) == 0);
        const float zero[VEC] = {};
        while (rows) {
            float* to = gW + (v0 + __builtin_ctzll(rows) / kSeek) * q.D;
            rows &= rows - 1;
            for (int d = lane * VEC; d < q.D; d += kWave * VEC) store_elems<float, VEC>(to + min(d, q.D - VEC), zero);
        }
        return;
    }
    const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int piece = __builtin_amdgcn_readfirstlane((int)(item / q.columns));
    const int column = __builtin_amdgcn_readfirstlane((int)(item - (int64_t)piece * q.columns));
    if (piece >= q.pieces) return;
    const int first = piece * q.piece, end = min((int64_t)first + q.piece, (int64_t)q.R);
    const int at = (column * kWave + lane) * VEC, d = min(at, q.D - VEC);
    const bool live = at < q.D;
    float acc[VEC];
#pragma unroll
    for (int k = 0; k < VEC; ++k) acc[k] = 0.0f;
    uint32_t run = uniform(keys[first]);
    bool open = first > 0 && uniform(keys[first - 1]) == run;      // the run comes from the piece before
    auto put = [&](float* to, float by) {
        float o[VEC];
#pragma unroll
        for (int k = 0; k < VEC; ++k) o[k] = acc[k] * by;
        if (live) store_elems<float, VEC>(to + d, o);
    };
    const int n = end - first;                                      // places near 2^31 are counted from the first
    for (int i0 = 0; i0 < n; i0 += kAhead) {
        E row[kAhead][VEC];
        uint32_t key[kAhead];
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            const int i = first + min(i0 + j, n - 1);
            key[j] = uniform(keys[i]);
            const int r = (int)uniform(places[i]), b = r / q.T;
            if (key[j] < (uint32_t)q.V)
                load_elems<E, VEC>(grad + b * q.g_batch + (r - b * q.T) * q.g_time + d, row[j]);
        }
#pragma unroll
        for (int j = 0; j < kAhead; ++j) {
            if (i0 + j >= n) break;
            if (key[j] != run) {
                if (open) put(part + (int64_t)piece * 2 * q.D, 1.0f);
                else put(gW + (int64_t)run * q.D, q.scale);
                run = key[j];
                open = false;
#pragma unroll
                for (int k = 0; k < VEC; ++k) acc[k] = 0.0f;
            }
            if (run >= (uint32_t)q.V) return;                       // padding comes last
#pragma unroll
            for (int k = 0; k < VEC; ++k) acc[k] += to_f32(row[j][k]);
        }
    }
    const bool on = end < q.R && uniform(keys[end]) == run;        // it goes on in the next piece
    if (open) {
        put(part + (int64_t)piece * 2 * q.D, 1.0f);
    } else if (on) {
        put(part + ((int64_t)piece * 2 + 1) * q.D, 1.0f);
        if (column == 0 && lane == 0) list[1 + atomicAdd(list, 1u)] = piece;
    } else {
        put(gW + (int64_t)run * q.D, q.scale);
    }
}

// A workgroup takes 64 VEC columns of a listed piece: the parts of the run that
// begins there are added up, each wave's share of the pieces in order.
template <int VEC>
__global__ __launch_bounds__(kJoinWaves* kWave) void k_embed_join(const uint32_t* __restrict__ keys, Sums q,
                                                                  const float* __restrict__ part,
                                                                  const uint32_t* __restrict__ list,
                                                                  float* __restrict__ gW)
{
    __shared__ float sh[kJoinWaves][kWave * VEC];
    const int lane = threadIdx.x & 63, w = threadIdx.x >> 6;
    const int64_t items = (int64_t)*list * q.columns;
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const int piece = (int)list[1 + item / q.columns], column = (int)(item % q.columns);
        const uint32_t run = keys[(int64_t)(piece + 1) * q.piece];
        int n = 2;                                                  // pieces that the run lies in
        for (;;) {
            const int64_t next = ((int64_t)piece + n + lane) * q.piece;
            const uint64_t on = __ballot(next < q.R && keys[min(next, (int64_t)q.R - 1)] == run);
            const int more = ~on ? __builtin_ctzll(~on) : kWave;
            n += more;
            if (more < kWave) break;
        }
        const int at = (column * kWave + lane) * VEC, d = min(at, q.D - VEC);
        float acc[VEC];
#pragma unroll
        for (int k = 0; k < VEC; ++k) acc[k] = 0.0f;
        const int to = (int)((int64_t)n * (w + 1) / kJoinWaves);
#pragma unroll 8
        for (int j = (int)((int64_t)n * w / kJoinWaves); j < to; ++j) {
            float v[VEC];
            load_elems<float, VEC>(part + ((int64_t)(piece + j) * 2 + (j == 0)) * q.D + d, v);
#pragma unroll
            for (int k = 0; k < VEC; ++k) acc[k] += v[k];
        }
#pragma unroll
        for (int k = 0; k < VEC; ++k) sh[w][lane * VEC + k] = acc[k];
        __syncthreads();
        if (w == 0 && at < q.D) {
#pragma unroll
            for (int k = 0; k < VEC; ++k) {
                acc[k] = 0.0f;
                for (int j = 0; j < kJoinWaves; ++j) acc[k] += sh[j][lane * VEC + k];
                acc[k] *= q.scale;
            }
            store_elems<float, VEC>(gW + (int64_t)run * q.D + d, acc);
        }
        __syncthreads();
    }
}

// No token at all: the gradient is 0.
__global__ __launch_bounds__(256) void k_clear(float* __restrict__ to, int64_t n)
{
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) to[i] = 0.0f;
}

int check_embed(const lif_embed_params* p)
{
    if (!p || p->B < 0 || p->T < 0 || p->V < 1 || p->D < 1 || p->flags != 0 || p->reserved != 0) return LIF_ERR_ARG;
    for (int t : {p->dtype, p->table})
        if (t != LIF_F32 && t != LIF_BF16 && t != LIF_F16) return LIF_ERR_ARG;
    if (p->w_row < p->D || p->g_batch < 0 || p->g_time < 0 || !isfinite(p->scale) || !isfinite((float)p->scale))
        return LIF_ERR_ARG;
    if (p->V > (1 << 24) || p->D > (1 << 20) || (int64_t)p->B * p->T >= ((int64_t)1 << 31)) return LIF_ERR_SIZE;
    return LIF_OK;
}

int vec_of(int D) { return D >= 4 ? 4 : 1; }

template <int V> struct Int { static constexpr int value = V; };

struct Plan {
    int passes, bits, chunk, chunks;
    Sums s;
    size_t keys[2], places[2], count, total, part, list, end;
};

Plan plan_of(const lif_embed_params& p)
{
    Plan q;
    const int R = p.B * p.T;
    int bits = 1;
    while (((int64_t)1 << bits) <= p.V) ++bits;                     // keys are 0 .. V
    q.passes = (bits + kMaxBits - 1) / kMaxBits;
    q.bits = (bits + q.passes - 1) / q.passes;
    const int64_t least = ((int64_t)R + kChunks - 1) / kChunks, unit = kSortWaves * kWave;
    q.chunk = (int)((least + unit - 1) / unit * unit);
    q.chunks = q.chunk ? (int)(((int64_t)R + q.chunk - 1) / q.chunk) : 0;
    Sums& s = q.s;
    s.R = R, s.T = p.T, s.V = p.V, s.D = p.D;
    s.columns = (p.D + kWave * vec_of(p.D) - 1) / (kWave * vec_of(p.D));
    s.g_batch = p.g_batch, s.g_time = p.g_time;
    s.scale = (float)p.scale;
    int64_t piece = ((int64_t)R * s.columns + 8191) / 8192;
    if (piece < 16) piece = 16;
    if (R <= 64) piece = 64;                                        // one piece: no join
    if (piece > 1 << 30) piece = 1 << 30;
    s.piece = (int)piece;
    s.pieces = (int)(((int64_t)R + piece - 1) / piece);
    size_t at = 0;
    auto take = [&](size_t bytes) {
        const size_t here = at;
        at += (bytes + 15) & ~(size_t)15;
        return here;
    };
    for (int i = 0; i < 2; ++i) {
        q.keys[i] = take(sizeof(uint32_t) * (size_t)R);
        q.places[i] = take(sizeof(uint32_t) * (size_t)R);
        if (q.passes == 1) q.keys[1] = q.keys[0], q.places[1] = q.places[0], i = 2;
    }
    q.count = take(sizeof(uint32_t) * ((size_t)q.chunks << q.bits));
    q.total = take(sizeof(uint32_t) << q.bits);
    q.part = take(sizeof(float) * 2 * (size_t)s.pieces * p.D);
    q.list = take(sizeof(uint32_t) * (1 + (size_t)s.pieces));
    q.end = R > 0 ? at : 0;
    return q;
}

}  // namespace
}  // namespace lif

extern "C" int lif_embed(const int32_t* token, const void* W, const int32_t* length, const lif_embed_params* p,
                         void* out, lif_stream_t stream)
{
    using namespace lif;
    const int rc = check_embed(p);
    if (rc) return rc;
    const int64_t R = (int64_t)p->B * p->T;
    if (R == 0) return LIF_OK;
    if (!token || !W || !out) return LIF_ERR_ARG;
    const int vec = vec_of(p->D), groups = (p->D + vec - 1) / vec;
    // a workgroup's rows: about 1024 vectors, and no more than 2^22 workgroups
    int rows = groups >= 1024 ? 1 : 1024 / groups;
    while ((R + rows - 1) / rows > (1 << 22)) rows *= 2;
    with_dtype(p->table, [&](auto e) {
        with_dtype(p->dtype, [&](auto f) {
            using E = decltype(e);
            using F = decltype(f);
            const dim3 grid((unsigned)((R + rows - 1) / rows));
            if (vec == 4)
                TIMED_LAUNCH("embed", (k_embed<E, F, 4>), grid, dim3(256), 0, (hipStream_t)stream, token, (const E*)W,
                             length, p->T, p->V, p->D, groups, rows, p->w_row, (float)p->scale, (int)R, (F*)out);
            else
                TIMED_LAUNCH("embed", (k_embed<E, F, 1>), grid, dim3(256), 0, (hipStream_t)stream, token, (const E*)W,
                             length, p->T, p->V, p->D, groups, rows, p->w_row, (float)p->scale, (int)R, (F*)out);
        });
    });
    return check_launch();
}

extern "C" size_t lif_embed_backward_workspace_size(const lif_embed_params* p)
{
    using namespace lif;
    if (check_embed(p) != LIF_OK) return 0;
    return plan_of(*p).end;
}

extern "C" int lif_embed_backward(const int32_t* token, const void* grad, const int32_t* length,
                                  const lif_embed_params* p, float* grad_W, void* ws, size_t ws_bytes,
                                  lif_stream_t stream)
{
    using namespace lif;
    const int rc = check_embed(p);
    if (rc) return rc;
    const int64_t R = (int64_t)p->B * p->T;
    if (!grad_W || (R > 0 && (!token || !grad))) return LIF_ERR_ARG;
    const Plan q = plan_of(*p);
    if (q.end > 0 && (!ws || (uintptr_t)ws % 16)) return LIF_ERR_ARG;
    if (ws_bytes < q.end) return LIF_ERR_WORKSPACE;
    const hipStream_t s = (hipStream_t)stream;
    if (R == 0) {
        TIMED_LAUNCH("embed_clear", k_clear, dim3(1024), dim3(256), 0, s, grad_W, (int64_t)p->V * p->D);
        return check_launch();
    }
    char* base = (char*)ws;
    uint32_t *count = (uint32_t*)(base + q.count), *total = (uint32_t*)(base + q.total);
    const uint32_t *keys = nullptr, *places = nullptr;
    uint32_t* list = (uint32_t*)(base + q.list);
    if (R <= kFew) {
        int bits = 1;
        while ((1 << bits) <= p->V) ++bits;
        const Sort o = {(int)R, p->T, p->V, 0, bits, 0};
        uint32_t *ko = (uint32_t*)(base + q.keys[0]), *po = (uint32_t*)(base + q.places[0]);
        TIMED_LAUNCH("embed_sort_few", k_sort_few, dim3(1), dim3(kSmallWaves * kWave), 0, s, token, length, o, ko, po,
                     list);
        keys = ko, places = po;
    }
    for (int i = 0; i < q.passes && R > kFew; ++i) {
        const Sort o = {(int)R, p->T, p->V, q.chunk, q.bits, i * q.bits};
        uint32_t *ko = (uint32_t*)(base + q.keys[i & 1]), *po = (uint32_t*)(base + q.places[i & 1]);
        const int bins = 1 << q.bits;
        TIMED_LAUNCH("embed_count", k_count, dim3(q.chunks), dim3(kSortWaves * kWave), 0, s, token, length, keys, o,
                     count);
        TIMED_LAUNCH("embed_chunks", k_chunk_sums, dim3((bins + kWave - 1) / kWave), dim3(16 * kWave), 0, s, count,
                     q.chunks, bins, total);
        TIMED_LAUNCH("embed_sort", k_hand_out, dim3(q.chunks), dim3(kSortWaves * kWave), 0, s, token, length, keys,
                     places, o, count, total, ko, po, list);
        keys = ko, places = po;
    }
    const int64_t items = (int64_t)q.s.pieces * q.s.columns, sum_blocks = (items + 3) / 4;
    const int64_t rows = 4 * kWave / kSeek, zero_blocks = ((int64_t)p->V + rows - 1) / rows;
    float* part = (float*)(base + q.part);
    with_dtype(p->dtype, [&](auto e) {
        using E = decltype(e);
        auto with = [&](auto vec) {
            constexpr int VEC = decltype(vec)::value;
            TIMED_LAUNCH("embed_sums", (k_embed_sums<E, VEC>), dim3((unsigned)(sum_blocks + zero_blocks)), dim3(256),
                         0, s, (const E*)grad, keys, places, q.s, sum_blocks, grad_W, part, list);
            if (q.s.pieces > 1)
                TIMED_LAUNCH("embed_join", (k_embed_join<VEC>), dim3((unsigned)(items < 1024 ? items : 1024)),
                             dim3(kJoinWaves * kWave), 0, s, keys, q.s, part, list, grad_W);
        };
        if (vec_of(p->D) == 4) with(Int<4>());
        else with(Int<1>());
    });
    return check_launch();
}
