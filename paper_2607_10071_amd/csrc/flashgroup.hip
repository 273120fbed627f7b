// Group norm with an activation on channels-last maps, and its gradients, for AMD MI355X
// (gfx950).  C ABI: include/block/flashlayer.h.
//
//   y = act((x - mean) rstd weight + bias), mean and rstd of a sample's positions and a group
//
// Memory bounds all of it (about 15 operations an element).  Statistics go over whole
// samples, so x is read twice; the second time the last-level cache (256 MiB) gives what it
// still holds.  A map is cut into chunks of rows; a lane takes 16 bytes of consecutive
// channels and every so-many-th row of its chunk.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "block/flashlayer.h"
#include "block_act.h"
#include "block_common.h"

namespace {

struct Group {
    const char *x, *gy;          // gy: the output's gradient
    char *y;                     // or grad_x
    const char *weight, *bias;   // null: 1 and 0
    char *gweight, *gbias;       // null: not wanted
    float *stats;                // [N][groups][2]
    // forward: [N][chunks][groups + slices][2], a mean and a sum of squared differences for
    // each group in each slice (at group + slice); backward: [N][chunks][2][C]
    float *partial;
    float *sums;                 // backward: [N][2][C], then [N][groups][2] means
    int64_t N, R, ldx, ldy;      // elements
    int64_t chunk;               // rows of a chunk
    int C, groups, per;          // per: channels of a group
    int chunks, slices;          // of rows; of columns
    int slice;                   // columns of a slice
    int param_f32;
    float eps;
};

template <int DT>
struct Lane {
    static constexpr int ES = elem_size(DT), V = 16 / ES;   // channels of a lane

    static __device__ __forceinline__ u32x4 load(const char *row, int c, int C)
    {
        return c + V <= C ? load16(row + c * ES) : load_granule_edge<DT>(row, c, C);
    }

    static __device__ __forceinline__ void floats(u32x4 raw, float (&v)[V])
    {
        const u32x4 r[1] = {raw};
        elems_of<DT>(r, v);
    }

    static __device__ __forceinline__ void store(char *row, int c, int end, const float (&v)[V])
    {
        if (c + V <= end) {
            store_elems<DT>(row + c * ES, v);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (c + i < end) store_elem<DT>(row, c + i, v[i]);
        }
    }
};

__device__ __forceinline__ float param(const char *p, int f32, int dt, int c, float otherwise)
{
    if (!p) return otherwise;
    if (f32 || dt == FLASHBEV_F32) return load_elem<FLASHBEV_F32>(p, c);
    return dt == FLASHBEV_F16 ? load_elem<FLASHBEV_F16>(p, c) : load_elem<FLASHBEV_BF16>(p, c);
}

__device__ __forceinline__ void put_param(char *p, int f32, int dt, int c, float v)
{
    if (f32 || dt == FLASHBEV_F32) {
        store_elem<FLASHBEV_F32>(p, c, v);
    } else if (dt == FLASHBEV_F16) {
        store_elem<FLASHBEV_F16>(p, c, v);
    } else {
        store_elem<FLASHBEV_BF16>(p, c, v);
    }
}

// (mean, sum of squared differences) of n values joined with those of m others.  No difference of
// large sums is taken.  The join's term d^2 carries the means' errors times 2 d, so means are kept
// relative to a value of the group itself (pivot, below), which an offset far above the spread
// leaves small.
__device__ __forceinline__ void join(float &mean, float &sq, float n, float mean2, float sq2, float m)
{
    const float tot = n + m;
    if (tot == 0.0f) return;
    const float d = mean2 - mean, share = m / tot;
    mean = __builtin_fmaf(d, share, mean);
    sq += __builtin_fmaf(d * d, n * share, sq2);
}

constexpr int kBatch = 8;   // rows of a lane that are in flight together

// The value that a group's means are relative to: the middle one of its first channel's at the first,
// middle and last position.  (The first alone cost the means 2^-24 of what it was away from the others.)
template <int DT>
__device__ __forceinline__ float pivot(const Group &p, int64_t n, int g)
{
    const char *x = p.x + n * p.R * p.ldx * elem_size(DT);
    return __builtin_amdgcn_fmed3f(load_elem<DT>(x, g * p.per), load_elem<DT>(x, (p.R - 1) / 2 * p.ldx + g * p.per),
                                   load_elem<DT>(x, (p.R - 1) * p.ldx + g * p.per));
}

// The pivots of a lane's channels, of which the last is end - 1.
template <int DT>
__device__ __forceinline__ void pivots(const Group &p, int64_t n, int c, int end, float (&from)[Lane<DT>::V])
{
    constexpr int V = Lane<DT>::V;
    if (p.per % V == 0) {   // (one group's)
        from[0] = pivot<DT>(p, n, c / p.per);
#pragma unroll
        for (int i = 1; i < V; ++i) from[i] = from[0];
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) from[i] = pivot<DT>(p, n, min(c + i, end - 1) / p.per);
    }
}

// Rows r, r + step, .. of a batch, in flight together: all eight, or the first `rows`.
template <int DT, class W>
__device__ __forceinline__ void load_batch(u32x4 (&raw)[kBatch], const char *x, int64_t ld, int64_t r, int64_t step,
                                           int rows, W whole, int c, int C)
{
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
        raw[b] = u32x4{0, 0, 0, 0};
        if (whole.value || b < rows) raw[b] = Lane<DT>::load(x + (r + b * step) * ld * Lane<DT>::ES, c, C);
    }
}

// A batch's means, from `from`, and sums of squared differences.
template <int DT, class W>
__device__ __forceinline__ void batch_stats(const u32x4 (&raw)[kBatch], int rows, W whole,
                                            const float (&from)[Lane<DT>::V], float (&s)[Lane<DT>::V],
                                            float (&q)[Lane<DT>::V])
{
    using L = Lane<DT>;
    float v[L::V];
#pragma unroll
    for (int i = 0; i < L::V; ++i) s[i] = q[i] = 0.0f;
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
        L::floats(raw[b], v);
#pragma unroll
        for (int i = 0; i < L::V; ++i) s[i] += whole.value || b < rows ? v[i] - from[i] : 0.0f;
    }
    const float share = whole.value ? 1.0f / kBatch : 1.0f / (float)rows;
#pragma unroll
    for (int i = 0; i < L::V; ++i) s[i] *= share;
#pragma unroll
    for (int b = 0; b < kBatch; ++b) {
        L::floats(raw[b], v);
#pragma unroll
        for (int i = 0; i < L::V; ++i) {
            const float d = whole.value || b < rows ? v[i] - from[i] - s[i] : 0.0f;
            q[i] = __builtin_fmaf(d, d, q[i]);
        }
    }
}

// A lane's channels over the rows r0, r0 + step, .. < r1: means, from their groups' pivots, and
// sums of squared differences; returns the number of rows.  Eight rows' mean and differences are
// formed in registers, then joined: 5 operations an element, where row by row would take 7 and a
// division.
template <int DT>
__device__ __forceinline__ float lane_stats(const Group &p, int64_t n_, int c, int C, int64_t r0, int64_t r1,
                                            int64_t step, float (&mean)[Lane<DT>::V], float (&sq)[Lane<DT>::V])
{
    using L = Lane<DT>;
    const char *x = p.x + n_ * p.R * p.ldx * L::ES;
    float n = 0.0f, from[L::V];
#pragma unroll
    for (int i = 0; i < L::V; ++i) mean[i] = sq[i] = 0.0f;
    pivots<DT>(p, n_, c, C, from);
    const auto batch = [&](int64_t r, int rows, auto whole) {
        u32x4 raw[kBatch];
        float s[L::V], q[L::V];
        load_batch<DT>(raw, x, p.ldx, r, step, rows, whole, c, C);
        batch_stats<DT>(raw, rows, whole, from, s, q);
#pragma unroll
        for (int i = 0; i < L::V; ++i) join(mean[i], sq[i], n, s[i], q[i], (float)rows);
        n += (float)rows;
    };
    int64_t r = r0;
    for (; r + (kBatch - 1) * step < r1; r += kBatch * step) batch(r, kBatch, std::true_type{});
    if (r < r1) batch(r, (int)((r1 - r + step - 1) / step), std::false_type{});
    return n;
}

// The (mean, squares, count) of `width` neighbouring lanes, a power of two; all end with the whole.
// Both sides of a pair join the same way round, so that all lanes agree.
__device__ __forceinline__ void wave_stats(float &mean, float &sq, float &n, int width = 64)
{
    for (int o = 1; o < width; o *= 2) {
        const float m2 = __shfl_xor(mean, o), s2 = __shfl_xor(sq, o), n2 = __shfl_xor(n, o);
        const bool low = !(threadIdx.x & o);
        float a = low ? mean : m2, b = low ? sq : s2, k = low ? n : n2;
        join(a, b, k, low ? m2 : mean, low ? s2 : sq, low ? n2 : n);
        mean = a;
        sq = b;
        n = n + n2;
    }
}

struct Place {   // a workgroup's sample, chunk of rows and slice of columns; a lane's column and row
    int64_t n, chunk, r0, r1;
    int c0, c1, vecs, cv, rr, rows;
};

template <int V>
__device__ __forceinline__ Place place_of(const Group &p, uint32_t id, int threads)
{
    Place l;
    const uint32_t s = id % p.slices;
    id /= p.slices;
    l.chunk = id % p.chunks;
    l.n = id / p.chunks;
    l.r0 = l.chunk * p.chunk;
    l.r1 = min(l.r0 + p.chunk, p.R);
    l.c0 = s * p.slice;
    l.c1 = min(l.c0 + p.slice, p.C);
    l.vecs = (l.c1 - l.c0 + V - 1) / V;
    l.rr = threadIdx.x / l.vecs;
    l.cv = threadIdx.x - l.rr * l.vecs;
    l.rows = min((int64_t)threads / l.vecs, l.r1 - l.r0);
    return l;
}

// The statistics of the groups that columns c0 .. c1 - 1 hold (parts of), of their channels' in
// `lds` (means, then sums of squared differences `vecs` * V further on), each of `rows` values.
// As many lanes to a group as it has channels, up to a wavefront; `put` gets the group, its
// mean, squares and count in one lane.  (The first pass of 139200 x 256 in 32 groups by 972
// workgroups: 25.6 us, 38 with a wavefront to each group of 8 channels.)
template <class F>
__device__ __forceinline__ void join_channels(const float *lds, int squares, int c0, int c1, int per, float rows,
                                              int waves, F put)
{
    int width = 1;
    while (width < per && width < 64) width *= 2;
    const int lane = threadIdx.x & (width - 1), g0 = c0 / per, each = waves * 64 / width;
    // (whole wavefronts go round together: their lanes exchange values)
    for (int base = g0; base * per < c1; base += each) {
        const int g = base + (int)threadIdx.x / width;
        float m = 0.0f, s = 0.0f, k = 0.0f;
        const int first = max(c0, g * per) - c0, last = min(c1, (g + 1) * per) - c0;
        for (int i = first + lane; i < last; i += width) {
            join(m, s, k, lds[i], lds[squares + i], rows);
            k += rows;
        }
        wave_stats(m, s, k, width);
        if (lane == 0 && first < last) put(g, m, s, k);
    }
}

// The channels' statistics of all lanes' of a column (l.rows of them): means in the first l.vecs V
// of `out`, then squares.  Up to a wavefront's lanes to a channel, which join the rows' lanes in
// turn and then each other.  (Six samples of 704 x 32 float32 in one launch: 8.8 us, 9.6 with a
// tree over the rows, which takes two barriers a level.)
template <int V, int THREADS>
__device__ __forceinline__ void channel_stats(float *lds, float *out, const Place &l, const float (&mean)[V],
                                              const float (&sq)[V], float n)
{
    constexpr int S = 2 * V + 1;
    if (l.rr < l.rows) {
        float *at = lds + (l.rr * l.vecs + l.cv) * S;
#pragma unroll
        for (int i = 0; i < V; ++i) {
            at[i] = mean[i];
            at[V + i] = sq[i];
        }
        at[2 * V] = n;
    }
    __syncthreads();
    const int channels = l.vecs * V;
    int width = 1;
    while (width < 64 && width < l.rows && 2 * width * channels <= THREADS) width *= 2;
    const int lane = threadIdx.x & (width - 1);
    // (whole wavefronts go round together: their lanes exchange values)
    for (int base = 0; base < channels; base += THREADS / width) {
        const int c = base + (int)threadIdx.x / width;
        float m = 0.0f, s = 0.0f, k = 0.0f;
        if (c < channels) {
            const float *at = lds + (lane * l.vecs + c / V) * S;
            for (int r = lane; r < l.rows; r += width, at += width * l.vecs * S) {
                join(m, s, k, at[c % V], at[V + c % V], at[2 * V]);
                k += at[2 * V];
            }
        }
        wave_stats(m, s, k, width);
        if (lane == 0 && c < channels) {
            out[c] = m;
            out[channels + c] = s;
        }
    }
    __syncthreads();
}

// First pass: each chunk's statistics of every group.
template <int DT>
__global__ void __launch_bounds__(256) group_stats(Group p)
{
    using L = Lane<DT>;
    __shared__ float lds[256 * (2 * L::V + 1)], channels[2 * 256 * L::V];
    const uint32_t id = block_index();
    if (id >= (uint64_t)p.N * p.chunks * p.slices) return;
    const Place l = place_of<L::V>(p, id, 256);
    float mean[L::V], sq[L::V], n = 0.0f;
    const int c = l.c0 + l.cv * L::V;
    if (l.rr < l.rows)
        n = lane_stats<DT>(p, l.n, c, l.c1, l.r0 + l.rr, l.r1, l.rows, mean, sq);
    channel_stats<L::V, 256>(lds, channels, l, mean, sq, n);
    float *o = p.partial + (l.n * p.chunks + l.chunk) * 2 * (p.groups + p.slices);
    const int s = l.c0 / p.slice;
    join_channels(channels, l.vecs * L::V, l.c0, l.c1, p.per, (float)(l.r1 - l.r0), 4, [&](int g, float m, float q, float) {
        o[2 * (g + s)] = m;
        o[2 * (g + s) + 1] = q;
    });
}

// A sample's and group's statistics of its chunks and slices: a workgroup.
template <int DT>
__global__ void __launch_bounds__(256) group_join(Group p)
{
    __shared__ float lds[4][3];
    const uint32_t id = block_index();
    if (id >= (uint64_t)p.N * p.groups) return;
    const int64_t n = id / p.groups;
    const int g = id - n * p.groups;
    float mean = 0.0f, sq = 0.0f, cnt = 0.0f;
    const int c0 = g * p.per, c1 = c0 + p.per;
    for (int s = c0 / p.slice; s * p.slice < c1; ++s) {
        const float width = (float)(min(c1, (s + 1) * p.slice) - max(c0, s * p.slice));
        for (int k = threadIdx.x; k < p.chunks; k += 256) {
            const float *o = p.partial + ((n * p.chunks + k) * (p.groups + p.slices) + g + s) * 2;
            const float m = (float)min(p.chunk, p.R - k * p.chunk) * width;
            join(mean, sq, cnt, o[0], o[1], m);
            cnt += m;
        }
    }
    wave_stats(mean, sq, cnt);
    if ((threadIdx.x & 63) == 0) {
        lds[threadIdx.x >> 6][0] = mean;
        lds[threadIdx.x >> 6][1] = sq;
        lds[threadIdx.x >> 6][2] = cnt;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 4; ++w) {
            join(mean, sq, cnt, lds[w][0], lds[w][1], lds[w][2]);
            cnt += lds[w][2];
        }
        p.stats[2 * (int64_t)id] = pivot<DT>(p, n, g) + mean;
        p.stats[2 * (int64_t)id + 1] = 1.0f / sqrtf(sq / cnt + p.eps);
    }
}

// A lane's channels' factors: xhat = (x - mean) rstd.
template <int DT>
struct Factors {
    static constexpr int V = Lane<DT>::V;
    float mean[V], rstd[V], w[V], b[V];

    __device__ __forceinline__ void load_params(const Group &p, int c, int end)
    {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int ci = min(c + i, end - 1);
            w[i] = param(p.weight, p.param_f32, DT, ci, 1.0f);
            b[i] = param(p.bias, p.param_f32, DT, ci, 0.0f);
        }
    }

    __device__ __forceinline__ void load_stats(const Group &p, const float *stats, int c, int end)
    {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const int g = min(c + i, end - 1) / p.per;
            mean[i] = stats[2 * g];
            rstd[i] = stats[2 * g + 1];
        }
    }

    __device__ __forceinline__ void load(const Group &p, const float *stats, int c, int end)
    {
        load_params(p, c, end);
        load_stats(p, stats, c, end);
    }

    // w becomes rstd weight
    __device__ __forceinline__ void fold()
    {
#pragma unroll
        for (int i = 0; i < V; ++i) w[i] *= rstd[i];
    }

    // A row's y, after fold().
    template <int ACT>
    __device__ __forceinline__ void put(char *y, u32x4 raw, int c, int end) const
    {
        float v[V];
        Lane<DT>::floats(raw, v);
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = act_value(ACT, __builtin_fmaf(v[i] - mean[i], w[i], b[i]));
        Lane<DT>::store(y, c, end, v);
    }
};

template <int DT, int ACT>
__device__ __forceinline__ void apply_rows(const Group &p, Factors<DT> &f, int64_t n, int c, int c1, int64_t r0,
                                           int64_t r1, int64_t step)
{
    using L = Lane<DT>;
    constexpr int U = 4;
    const char *x = p.x + n * p.R * p.ldx * L::ES;
    char *y = p.y + n * p.R * p.ldy * L::ES;
    f.fold();
    for (int64_t r = r0; r < r1; r += U * step) {
        u32x4 raw[U];
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (r + u * step < r1) raw[u] = L::load(x + (r + u * step) * p.ldx * L::ES, c, p.C);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            if (r + u * step >= r1) break;
            f.template put<ACT>(y + (r + u * step) * p.ldy * L::ES, raw[u], c, c1);
        }
    }
}

// Second pass: y.
template <int DT, int ACT>
__global__ void __launch_bounds__(256) group_apply(Group p)
{
    using L = Lane<DT>;
    const uint32_t id = block_index();
    if (id >= (uint64_t)p.N * p.chunks * p.slices) return;
    const Place l = place_of<L::V>(p, id, 256);
    if (l.rr >= l.rows) return;
    const int c = l.c0 + l.cv * L::V;
    Factors<DT> f;
    f.load(p, p.stats + 2 * l.n * p.groups, c, l.c1);
    apply_rows<DT, ACT>(p, f, l.n, c, l.c1, l.r0 + l.rr, l.r1, l.rows);
}

// Both passes by one workgroup for a sample's slice of whole groups, of up to eight rows a lane,
// which stay in registers between them (small maps: one launch in place of three).
constexpr int kWhole = 512;

template <int DT, int ACT>
__global__ void __launch_bounds__(kWhole) group_whole(Group p)
{
    using L = Lane<DT>;
    __shared__ float lds[kWhole * (2 * L::V + 1)], channels[2 * (kWhole + L::V)];
    __shared__ float stats[2 * kWhole];   // of the slice's groups
    const uint32_t id = block_index();
    if (id >= (uint64_t)p.N * p.slices) return;
    const int64_t n = id / p.slices;
    Place l;
    l.c0 = (id - (uint32_t)n * p.slices) * p.slice;
    l.c1 = min(l.c0 + p.slice, p.C);
    l.vecs = (l.c1 - l.c0 + L::V - 1) / L::V;
    l.rr = threadIdx.x / l.vecs;
    l.cv = threadIdx.x - l.rr * l.vecs;
    const int R = (int)p.R;
    l.rows = min(kWhole / l.vecs, R);
    const int c = l.c0 + l.cv * L::V, mine = l.rr < l.rows ? (R - l.rr + l.rows - 1) / l.rows : 0;
    u32x4 raw[kBatch];
    load_batch<DT>(raw, p.x + n * p.R * p.ldx * L::ES, p.ldx, l.rr, l.rows, mine, std::false_type{}, c, l.c1);
    Factors<DT> f;
    f.load_params(p, c, l.c1);
    float mean[L::V], sq[L::V], from[L::V], count = (float)mine;
    pivots<DT>(p, n, c, l.c1, from);
    batch_stats<DT>(raw, max(mine, 1), std::false_type{}, from, mean, sq);
    channel_stats<L::V, kWhole>(lds, channels, l, mean, sq, count);
    const int g0 = l.c0 / p.per;
    join_channels(channels, l.vecs * L::V, l.c0, l.c1, p.per, (float)R, kWhole / 64,
                  [&](int g, float m, float q, float k) {
                      const float r = 1.0f / sqrtf(q / k + p.eps);
                      m += pivot<DT>(p, n, g);
                      stats[2 * (g - g0)] = m;
                      stats[2 * (g - g0) + 1] = r;
                      if (p.stats) {
                          float *o = p.stats + 2 * (n * p.groups + g);
                          o[0] = m;
                          o[1] = r;
                      }
                  });
    __syncthreads();
    f.load_stats(p, stats - 2 * g0, c, l.c1);
    f.fold();
    char *y = p.y + (n * p.R + l.rr) * p.ldy * L::ES;
#pragma unroll
    for (int b = 0; b < kBatch; ++b)
        if (b < mine) f.template put<ACT>(y + (int64_t)b * l.rows * p.ldy * L::ES, raw[b], c, l.c1);
}

// ---------------------------------------------------------------------------
// backward
// ---------------------------------------------------------------------------
// First pass: each chunk's sums of d and d xhat for every channel.
template <int DT, int ACT>
__global__ void __launch_bounds__(256) group_sums(Group p)
{
    using L = Lane<DT>;
    constexpr int U = 4;
    __shared__ float lds[256 * (2 * L::V + 1)];
    const uint32_t id = block_index();
    if (id >= (uint64_t)p.N * p.chunks * p.slices) return;
    const Place l = place_of<L::V>(p, id, 256);
    const int c = l.c0 + l.cv * L::V;
    float s1[L::V], s2[L::V];
#pragma unroll
    for (int i = 0; i < L::V; ++i) s1[i] = s2[i] = 0.0f;
    if (l.rr < l.rows) {
        Factors<DT> f;
        f.load(p, p.stats + 2 * l.n * p.groups, c, l.c1);
        const char *x = p.x + l.n * p.R * p.ldx * L::ES, *gy = p.gy + l.n * p.R * p.ldy * L::ES;
        for (int64_t r = l.r0 + l.rr; r < l.r1; r += U * l.rows) {
            u32x4 rx[U], rg[U];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                rx[u] = rg[u] = u32x4{0, 0, 0, 0};
                const int64_t ru = r + u * l.rows;
                if (ru < l.r1) {
                    rx[u] = L::load(x + ru * p.ldx * L::ES, c, p.C);
                    rg[u] = L::load(gy + ru * p.ldy * L::ES, c, p.C);
                }
            }
#pragma unroll
            for (int u = 0; u < U; ++u) {
                if (r + u * l.rows >= l.r1) break;
                float v[L::V], d[L::V];
                L::floats(rx[u], v);
                L::floats(rg[u], d);
#pragma unroll
                for (int i = 0; i < L::V; ++i) {
                    const float h = (v[i] - f.mean[i]) * f.rstd[i];
                    if (ACT != FLASHBLOCK_ACT_NONE) d[i] *= act_slope(ACT, __builtin_fmaf(h, f.w[i], f.b[i]));
                    s1[i] += d[i];
                    s2[i] = __builtin_fmaf(d[i], h, s2[i]);
                }
            }
        }
    }
    float *at = lds + (l.rr * l.vecs + l.cv) * (2 * L::V + 1);
    for (int left = l.rows; left > 1;) {
        const int half = (left + 1) / 2;
        if (l.rr >= half && l.rr < left) {
#pragma unroll
            for (int i = 0; i < L::V; ++i) {
                at[i] = s1[i];
                at[L::V + i] = s2[i];
            }
        }
        __syncthreads();
        if (l.rr + half < left) {
            const float *o = at + half * l.vecs * (2 * L::V + 1);
#pragma unroll
            for (int i = 0; i < L::V; ++i) {
                s1[i] += o[i];
                s2[i] += o[L::V + i];
            }
        }
        __syncthreads();
        left = half;
    }
    if (l.rr == 0) {
        float *o = p.partial + (l.n * p.chunks + l.chunk) * 2 * p.C;
#pragma unroll
        for (int i = 0; i < L::V; ++i)
            if (c + i < l.c1) {
                o[c + i] = s1[i];
                o[p.C + c + i] = s2[i];
            }
    }
}

// A sample's sums of its chunks, for each channel: 32 channels and 32 shares of the chunks to a
// workgroup.
__global__ void __launch_bounds__(1024) group_sums_join(Group p)
{
    __shared__ float lds[2][32][33];
    const uint32_t blocks = (p.C + 31) / 32, id = block_index();
    if (id >= (uint64_t)p.N * blocks) return;
    const int64_t n = id / blocks;
    const int lane = threadIdx.x & 31, way = threadIdx.x >> 5, c = (id - n * blocks) * 32 + lane;
    float s1 = 0.0f, s2 = 0.0f;
    if (c < p.C) {
#pragma unroll 4
        for (int k = way; k < p.chunks; k += 32) {
            const float *o = p.partial + (n * p.chunks + k) * 2 * p.C;
            s1 += o[c];
            s2 += o[p.C + c];
        }
    }
    lds[0][way][lane] = s1;
    lds[1][way][lane] = s2;
    __syncthreads();
    for (int half = 16; half > 0; half /= 2) {
        if (way < half) {
            lds[0][way][lane] += lds[0][way + half][lane];
            lds[1][way][lane] += lds[1][way + half][lane];
        }
        __syncthreads();
    }
    if (way == 0 && c < p.C) {
        p.sums[2 * n * p.C + c] = lds[0][0][lane];
        p.sums[(2 * n + 1) * p.C + c] = lds[1][0][lane];
    }
}

// A sample's and group's means of d weight and d weight xhat: a wavefront.
template <int DT>
__global__ void __launch_bounds__(64) group_means(Group p)
{
    const uint32_t id = block_index();
    if (id >= (uint64_t)p.N * p.groups) return;
    const int64_t n = id / p.groups;
    const int g = id - n * p.groups;
    float t1 = 0.0f, t2 = 0.0f;
    for (int i = threadIdx.x; i < p.per; i += 64) {
        const int c = g * p.per + i;
        const float w = param(p.weight, p.param_f32, DT, c, 1.0f);
        t1 = __builtin_fmaf(w, p.sums[2 * n * p.C + c], t1);
        t2 = __builtin_fmaf(w, p.sums[(2 * n + 1) * p.C + c], t2);
    }
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
        t1 += __shfl_xor(t1, o);
        t2 += __shfl_xor(t2, o);
    }
    if (threadIdx.x == 0) {
        float *o = p.sums + 2 * p.N * p.C + 2 * (int64_t)id;
        const float count = (float)p.R * (float)p.per;
        o[0] = t1 / count;
        o[1] = t2 / count;
    }
}

// Second pass: grad_x, and by the workgroups past those of the map the sums over samples for
// weight and bias.
template <int DT, int ACT>
__global__ void __launch_bounds__(256) group_grad(Group p)
{
    using L = Lane<DT>;
    constexpr int U = 4;
    const uint32_t id = block_index();
    const uint64_t map = p.y ? (uint64_t)p.N * p.chunks * p.slices : 0;
    if (id >= map) {
        const uint64_t c = (id - map) * 256 + threadIdx.x;
        if (c >= (uint64_t)p.C) return;
        float s1 = 0.0f, s2 = 0.0f;
        for (int64_t n = 0; n < p.N; ++n) {
            s1 += p.sums[2 * n * p.C + c];
            s2 += p.sums[(2 * n + 1) * p.C + c];
        }
        if (p.gweight) put_param(p.gweight, p.param_f32, DT, (int)c, s2);
        if (p.gbias) put_param(p.gbias, p.param_f32, DT, (int)c, s1);
        return;
    }
    const Place l = place_of<L::V>(p, id, 256);
    if (l.rr >= l.rows) return;
    const int c = l.c0 + l.cv * L::V;
    Factors<DT> f;
    f.load(p, p.stats + 2 * l.n * p.groups, c, l.c1);
    float m1[L::V], m2[L::V];
    const float *means = p.sums + 2 * p.N * p.C + 2 * l.n * p.groups;
#pragma unroll
    for (int i = 0; i < L::V; ++i) {
        const int g = min(c + i, l.c1 - 1) / p.per;
        m1[i] = means[2 * g];
        m2[i] = means[2 * g + 1];
    }
    const char *x = p.x + l.n * p.R * p.ldx * L::ES, *gy = p.gy + l.n * p.R * p.ldy * L::ES;
    char *o = p.y + l.n * p.R * p.C * L::ES;
    for (int64_t r = l.r0 + l.rr; r < l.r1; r += U * l.rows) {
        u32x4 rx[U], rg[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            rx[u] = rg[u] = u32x4{0, 0, 0, 0};
            const int64_t ru = r + u * l.rows;
            if (ru < l.r1) {
                rx[u] = L::load(x + ru * p.ldx * L::ES, c, p.C);
                rg[u] = L::load(gy + ru * p.ldy * L::ES, c, p.C);
            }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t ru = r + u * l.rows;
            if (ru >= l.r1) break;
            float v[L::V], d[L::V];
            L::floats(rx[u], v);
            L::floats(rg[u], d);
#pragma unroll
            for (int i = 0; i < L::V; ++i) {
                const float h = (v[i] - f.mean[i]) * f.rstd[i];
                if (ACT != FLASHBLOCK_ACT_NONE) d[i] *= act_slope(ACT, __builtin_fmaf(h, f.w[i], f.b[i]));
                v[i] = f.rstd[i] * __builtin_fmaf(-h, m2[i], __builtin_fmaf(d[i], f.w[i], -m1[i]));
            }
            L::store(o + ru * p.C * L::ES, c, l.c1, v);
        }
    }
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
int check(const flashlayer_group_norm *a)
{
    if (!a) return FLASHBEV_ERR_NULLPTR;
    if (a->N < 0 || a->R < 0 || a->C < 0 || a->groups < 1 || a->C % a->groups || a->ldx < a->C || a->ldy < a->C)
        return FLASHBEV_ERR_SHAPE;
    if (!known_dtype(a->dtype)) return FLASHBEV_ERR_DTYPE;
    if (a->param_dtype != a->dtype && a->param_dtype != FLASHBEV_F32) return FLASHBEV_ERR_DTYPE;
    if (a->act < FLASHBLOCK_ACT_NONE || a->act > FLASHBLOCK_ACT_SILU) return FLASHBEV_ERR_VALUE;
    if (!(a->eps > 0.0f) || !finite_value(a->eps)) return FLASHBEV_ERR_VALUE;
    if (a->C > FLASHBLOCK_NORM_MAX || a->ldx > FLASHBLOCK_LD_MAX || a->ldy > FLASHBLOCK_LD_MAX ||
        size_prod({(uint64_t)a->N, (uint64_t)a->R}) > FLASHBLOCK_ROWS_MAX)
        return FLASHBEV_ERR_UNSUPPORTED;
    return FLASHBEV_OK;
}

// How a call is cut.  Chunks of rows: a lane's batch of eight rows at least, and more where that
// would be over 768 workgroups, the three of a CU that run at once in the backward (139200 x 256
// bf16, a training step's first and second backward passes: 33 + 39 us,
// 45 + 48 of 972, 39 + 40 of 498).
struct Cut {
    bool whole;
    int slices, slice, chunks;
    int64_t chunk;
};

Cut cut(const flashlayer_group_norm *a, bool backward)
{
    const int es = elem_size(a->dtype), V = 16 / es, per = a->C / a->groups;
    Cut c{};
    // whole groups of 64 bytes or more to one workgroup, eight rows at most to its lanes (six samples
    // of 704 x 32 float32 8.9 us a call, 13.9 in three launches; eight of 128 x 1024 bf16 9.5 and 20.5)
    const int some = std::min(((64 / es + per - 1) / per) * per, a->C);
    if (!backward && some <= kWhole && a->R <= kBatch * (kWhole / ((some + V - 1) / V))) {
        c.whole = true;
        c.slice = some;
        c.slices = (a->C + c.slice - 1) / c.slice;
        c.chunks = 1;
        c.chunk = a->R;
        return c;
    }
    c.slice = std::min(a->C, 256 * V);
    c.slices = (a->C + c.slice - 1) / c.slice;
    const int64_t rows = 256 / ((c.slice + V - 1) / V);   // that the workgroup's lanes take at once
    const int64_t most = std::max<int64_t>(1, 768 / std::max<int64_t>(1, a->N * c.slices));
    c.chunk = std::max(rows * kBatch, ((a->R + most - 1) / most + rows - 1) / rows * rows);
    c.chunks = (int)((a->R + c.chunk - 1) / c.chunk);
    return c;
}

uint64_t round256(uint64_t v) { return (v + 255) & ~255ull; }

uint64_t partial_bytes(const flashlayer_group_norm *a, const Cut &c, bool backward)
{
    return round256((uint64_t)a->N * c.chunks * 2 * (backward ? a->C : a->groups + c.slices) * 4);
}

uint64_t forward_bytes(const flashlayer_group_norm *a)
{
    if (!a->N || !a->R || !a->C) return 0;   // (there is nothing to cut)
    const Cut c = cut(a, false);
    if (c.whole) return 0;
    return partial_bytes(a, c, false) + round256((uint64_t)a->N * a->groups * 8);
}

uint64_t backward_bytes(const flashlayer_group_norm *a)
{
    if (!a->N || !a->R || !a->C) return 0;
    return partial_bytes(a, cut(a, true), true) + round256((uint64_t)a->N * 2 * ((uint64_t)a->C + a->groups) * 4);
}

Group group_of(const flashlayer_group_norm *a, const Cut &c)
{
    Group p{};
    p.N = a->N;
    p.R = a->R;
    p.ldx = a->ldx;
    p.ldy = a->ldy;
    p.C = a->C;
    p.groups = a->groups;
    p.per = a->C / a->groups;
    p.chunk = c.chunk;
    p.chunks = c.chunks;
    p.slices = c.slices;
    p.slice = c.slice;
    p.param_f32 = a->param_dtype == FLASHBEV_F32;
    p.eps = a->eps;
    return p;
}

#define BY_ACT(KERNEL, DT)                                                                   \
    (act == FLASHBLOCK_ACT_RELU        ? (const void *)KERNEL<DT, FLASHBLOCK_ACT_RELU>       \
     : act == FLASHBLOCK_ACT_GELU      ? (const void *)KERNEL<DT, FLASHBLOCK_ACT_GELU>       \
     : act == FLASHBLOCK_ACT_GELU_TANH ? (const void *)KERNEL<DT, FLASHBLOCK_ACT_GELU_TANH>  \
     : act == FLASHBLOCK_ACT_SILU      ? (const void *)KERNEL<DT, FLASHBLOCK_ACT_SILU>       \
                                       : (const void *)KERNEL<DT, FLASHBLOCK_ACT_NONE>)
#define BY_TYPE_AND_ACT(KERNEL)                                       \
    (dt == FLASHBEV_F32   ? BY_ACT(KERNEL, FLASHBEV_F32)              \
     : dt == FLASHBEV_F16 ? BY_ACT(KERNEL, FLASHBEV_F16)              \
                          : BY_ACT(KERNEL, FLASHBEV_BF16))
#define BY_TYPE(KERNEL)                                               \
    (dt == FLASHBEV_F32   ? (const void *)KERNEL<FLASHBEV_F32>        \
     : dt == FLASHBEV_F16 ? (const void *)KERNEL<FLASHBEV_F16>        \
                          : (const void *)KERNEL<FLASHBEV_BF16>)

struct Range {
    const void *p;
    uint64_t n;
};

int check_ranges(std::initializer_list<Range> outs, std::initializer_list<Range> ins)
{
    for (const Range *o = outs.begin(); o != outs.end(); ++o) {
        for (const Range &i : ins)
            if (ranges_overlap(o->p, o->n, i.p, i.n)) return FLASHBEV_ERR_ALIAS;
        for (const Range *q = outs.begin(); q != o; ++q)
            if (ranges_overlap(o->p, o->n, q->p, q->n)) return FLASHBEV_ERR_ALIAS;
    }
    return FLASHBEV_OK;
}

int check_workspace(const void *ws, uint64_t bytes, uint64_t need)
{
    if (!need) return FLASHBEV_OK;
    if (!ws) return FLASHBEV_ERR_NULLPTR;
    if (misaligned(ws, 256)) return FLASHBEV_ERR_ALIGN;
    return bytes < need ? FLASHBEV_ERR_SCRATCH : FLASHBEV_OK;
}

}  // namespace

extern "C" int flashlayer_group_norm_workspace_size(const flashlayer_group_norm *args, uint64_t *bytes)
{
    if (!bytes) return FLASHBEV_ERR_NULLPTR;
    if (const int rc = check(args)) return rc;
    *bytes = forward_bytes(args);
    return FLASHBEV_OK;
}

extern "C" int flashlayer_group_norm_backward_workspace_size(const flashlayer_group_norm *args, uint64_t *bytes)
{
    if (!bytes) return FLASHBEV_ERR_NULLPTR;
    if (const int rc = check(args)) return rc;
    *bytes = backward_bytes(args);
    return FLASHBEV_OK;
}

extern "C" int flashlayer_group_norm_forward(const flashlayer_group_norm *args, const void *x,
                                             const void *weight, const void *bias, void *y, float *stats,
                                             void *workspace, uint64_t workspace_bytes, void *stream)
{
    if (const int rc = check(args)) return rc;
    if (!args->N || !args->R || !args->C) return FLASHBEV_OK;
    const int dt = args->dtype, act = args->act, es = elem_size(dt), ps = elem_size(args->param_dtype);
    const int64_t M = args->N * args->R;
    const uint64_t need = forward_bytes(args);
    if (!x || !y) return FLASHBEV_ERR_NULLPTR;
    if (misaligned(x, es) || misaligned(y, es) || misaligned(weight, ps) || misaligned(bias, ps) ||
        misaligned(stats, 4))
        return FLASHBEV_ERR_ALIGN;
    if (const int rc = check_workspace(workspace, workspace_bytes, need)) return rc;
    const uint64_t vec = (uint64_t)args->C * ps;
    if (const int rc = check_ranges({{y, span_bytes(M, args->ldy, args->C, es)},
                                     {stats, (uint64_t)args->N * args->groups * 8},
                                     {workspace, need}},
                                    {{x, span_bytes(M, args->ldx, args->C, es)}, {weight, vec}, {bias, vec}}))
        return rc;
    const Cut c = cut(args, false);
    Group p = group_of(args, c);
    p.x = static_cast<const char *>(x);
    p.y = static_cast<char *>(y);
    p.weight = static_cast<const char *>(weight);
    p.bias = static_cast<const char *>(bias);
    p.stats = stats;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (c.whole) return launch_rows(BY_TYPE_AND_ACT(group_whole), (uint64_t)args->N * c.slices, kWhole, p, st);
    p.partial = static_cast<float *>(workspace);
    if (!stats) p.stats = reinterpret_cast<float *>(static_cast<char *>(workspace) + partial_bytes(args, c, false));
    const uint64_t blocks = (uint64_t)args->N * c.chunks * c.slices;
    if (const int rc = launch_rows(BY_TYPE(group_stats), blocks, 256, p, st)) return rc;
    if (const int rc = launch_rows(BY_TYPE(group_join), (uint64_t)args->N * args->groups, 256, p, st)) return rc;
    return launch_rows(BY_TYPE_AND_ACT(group_apply), blocks, 256, p, st);
}

extern "C" int flashlayer_group_norm_backward(const flashlayer_group_norm *args, const void *grad_y,
                                              const void *x, const float *stats, const void *weight,
                                              const void *bias, void *grad_x, void *grad_weight,
                                              void *grad_bias, void *workspace, uint64_t workspace_bytes,
                                              void *stream)
{
    if (const int rc = check(args)) return rc;
    const int dt = args->dtype, act = args->act, es = elem_size(dt), ps = elem_size(args->param_dtype);
    const int64_t M = args->N * args->R;
    const uint64_t need = backward_bytes(args), vec = (uint64_t)args->C * ps;
    if (!args->C) return FLASHBEV_OK;
    // (a gradient without elements may be null)
    if (!grad_x && !grad_weight && !grad_bias) return M ? FLASHBEV_ERR_NULLPTR : FLASHBEV_OK;
    if (misaligned(grad_weight, ps) || misaligned(grad_bias, ps)) return FLASHBEV_ERR_ALIGN;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    const uint64_t extra = grad_weight || grad_bias ? ((uint64_t)args->C + 255) / 256 : 0;
    if (M && (!grad_y || !x || !stats)) return FLASHBEV_ERR_NULLPTR;
    if (M && (misaligned(grad_y, es) || misaligned(x, es) || misaligned(stats, 4) || misaligned(weight, ps) ||
              misaligned(bias, ps) || misaligned(grad_x, es)))
        return FLASHBEV_ERR_ALIGN;
    if (const int rc = check_workspace(workspace, workspace_bytes, need)) return rc;
    const uint64_t rows_x = span_bytes(M, args->ldx, args->C, es), rows_g = span_bytes(M, args->ldy, args->C, es);
    if (const int rc = check_ranges({{grad_x, span_bytes(M, args->C, args->C, es)},
                                     {grad_weight, vec},
                                     {grad_bias, vec},
                                     {workspace, need}},
                                    {{grad_y, rows_g},
                                     {x, rows_x},
                                     {stats, (uint64_t)args->N * args->groups * 8},
                                     {weight, vec},
                                     {bias, vec}}))
        return rc;
    const Cut c = cut(args, true);
    Group p = group_of(args, c);
    p.weight = static_cast<const char *>(weight);
    p.bias = static_cast<const char *>(bias);
    p.gweight = static_cast<char *>(grad_weight);
    p.gbias = static_cast<char *>(grad_bias);
    if (!M) {   // no rows: the vectors' gradients are zeros
        p.N = 0;
        return launch_rows(BY_TYPE_AND_ACT(group_grad), extra, 256, p, st);
    }
    p.x = static_cast<const char *>(x);
    p.gy = static_cast<const char *>(grad_y);
    p.y = static_cast<char *>(grad_x);
    p.stats = const_cast<float *>(stats);
    p.partial = static_cast<float *>(workspace);
    p.sums = reinterpret_cast<float *>(static_cast<char *>(workspace) + partial_bytes(args, c, true));
    const uint64_t blocks = (uint64_t)args->N * c.chunks * c.slices;
    if (const int rc = launch_rows(BY_TYPE_AND_ACT(group_sums), blocks, 256, p, st)) return rc;
    if (const int rc = launch_rows((const void *)group_sums_join, (uint64_t)args->N * ((args->C + 31) / 32), 1024, p, st))
        return rc;
    if (grad_x)
        if (const int rc = launch_rows(BY_TYPE(group_means), (uint64_t)args->N * args->groups, 64, p, st)) return rc;
    return launch_rows(BY_TYPE_AND_ACT(group_grad), (grad_x ? blocks : 0) + extra, 256, p, st);
}
