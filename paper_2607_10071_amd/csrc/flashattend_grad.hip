// The gradients of attention, for AMD MI355X (gfx950).  C ABI: include/block/flashlayer.h; what
// the forward shares: flashattend.h.
//
// With p = exp(s - m) / l of the stored row statistics and dS = p (g v^T - delta),
// delta = g . out (g the output's gradient),
//
//   grad_q = scale dS k,   grad_k = scale dS^T q,   grad_v = p^T g
//
// Two kernels form the scores again, seven products in all: one with rows across sums grad_q
// over the keys, one with keys across sums grad_k and grad_v over the rows.  Five products
// in one kernel would leave grad_q to float atomics, whose order changes results.
//
// Digits.  p and dS are rounded to the inputs' type for their products: 900 x 40000 of 8 heads x 32 bf16 has
// grad_q off by 0.0025 of its norm, where the rounding of grad_q itself makes 0.0017, that of dS another 0.0018
// and the forward's rounded weights, in delta, 0.0005.  (dS in two terms would take 14 to 18% more of grad_q's
// kernel.)  bfloat16 has float32's
// range; float16 loses digits below 6e-5, where weights of one in 40000 and scaled losses'
// gradients lie, so its factors are kept near one: grad_q's kernel takes p l (at most 2^6) and
// g / (8 |g|), a row's factors coming back at the end; the other one takes p and dS times powers of
// two that bring the largest 1 / l and |g| / l of its rows to about one.  Both divide by one more for each
// power of two of |v| above 2^11, of a problem's largest or of each key's own (`spread`).
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "flashattend.h"

namespace {

// A row as the two kernels read it.
struct RowData {
    float m;       // its scores' reference; 0 for an empty row
    float log2l;   // of the sum of exp(s - m); infinite for an empty row, whose weights are then 0
    float delta;   // g . out
    float norm;    // float16: |g|
};

// an exponent whose power is a normal float32
__device__ __forceinline__ float within_range(float e)
{
    return __builtin_fminf(__builtin_fmaxf(e, -100.0f), 100.0f);
}

struct Backward : Attend {
    const char *out, *rest;   // [B, Lq, H, D]; rest null: none
    const float *stats;
    RowData *data;            // [B Hk][rows]
    float *largest;           // float16: [B Hk][padded / 16][3], the largest 1 / l, |g| / l and |out| of 16 rows
    // [B Hk][padded rows] each, for grad_k's and grad_v's kernel without masks: the exponent that a
    // row's weights lose, m log2(e) + log2(l), infinite past the last row; and delta
    float *lose, *delta;
    int padded;               // rows of a problem there: a multiple of 128
    char *gq, *gk, *gv;       // contiguous; null: not wanted
    float *part;              // splits > 1: grad_q's [splits][B Hk rows][DP] or
                              // grad_k's and grad_v's [2][splits][B Hk Lk][DP]
    int row_tiles;            // of 16
    uint32_t row_blocks;      // of all problems
    float *most_v;            // float16: [B Hk][key_tiles], the largest |v| of key_tile keys each
    int key_tiles, key_tile;  // 0 for other types
    uint32_t blocks_v;
    // q's and g's rows as grad_k's and grad_v's kernel without masks reads them: row r of head g of the
    // states at g `group` + (r / rshare) `row` + (r % rshare) `head`, of Dr channels
    const char *rq, *rg;
    int64_t rq_b, rq_g, rq_r, rq_h, rg_b, rg_g, rg_r, rg_h;
    int rshare, Dr;

    __device__ __forceinline__ void part_of(int r, int &i, int &j) const
    {
        if (rshare > 1) {
            row(r, i, j);
        } else {
            i = r;
            j = 0;
        }
    }
};

constexpr int kRowTile = 16;
constexpr int kMostTiles = 256;   // of largest |v|: four loads of a wavefront

// How many powers of two float16's dS is made smaller by for large values.  Weights p l reach 2^6 (a
// forward's reference may lag so far) and |g v^T - delta| is at most |g| (|v| + |out|): an eighth of one for
// |g| keeps their product within 2^15 up to |v| + |out| = 2^12, and each power of two above that takes another
// one.  (float16's largest, in 128 channels, takes 9; what is infinite makes dS what it makes it.)
__device__ __forceinline__ int spread(float sizes)
{
    int e = 0;
    while (e < 9 && sizes > (float)(4096 << e)) ++e;
    return e;
}

// The same by a problem's largest |v|, which no |out| passes.
__device__ __forceinline__ int spread_of_values(const Backward &p, int64_t problem, int lane)
{
    float most = 0.0f;
#pragma unroll
    for (int i = lane; i < lane + kMostTiles; i += 64)
        if (i < p.key_tiles) most = __builtin_fmaxf(most, p.most_v[problem * p.key_tiles + i]);
#pragma unroll
    for (int o = 1; o < 64; o *= 2) most = __builtin_fmaxf(most, __shfl_xor(most, o));
    return spread(2.0f * most);
}

// The same by a key's |v|, of its lane's fragments and the other half's, and its rows' largest |out|.
template <int N>
__device__ __forceinline__ int spread_of_key(const u32x4 (&vf)[N], float most_out)
{
    float sq = 0.0f;
#pragma unroll
    for (int c = 0; c < N; ++c) {
        const u32x4 w[1] = {vf[c]};
        float v[8];
        elems_of<FLASHBEV_F16>(w, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) sq = __builtin_fmaf(v[i], v[i], sq);
    }
    return spread(sqrtf(both_sum(sq)) + most_out);
}

// What a row's dS is multiplied by for grad_q's product.  float16 alone needs it: bfloat16 and float32
// hold what |g| makes of dS, and |g| itself would be squared beyond float32's range.
template <int DT>
__device__ __forceinline__ float row_factor(const Backward &p, const RowData &row, int64_t problem, int lane)
{
    if constexpr (DT == FLASHBEV_F16) {
        const float least = __builtin_ldexpf(0.125f, -spread_of_values(p, problem, lane));
        return row.norm > 0.0f ? least / row.norm : 1.0f;
    }
    return 1.0f;
}

// The largest |v| of a tile of keys, a lane to a granule of a key and four keys of its in flight.  (Copies are
// whole granules; masks that differ from row to row leave odd ones.)
template <int DT>
__device__ __forceinline__ void largest_values(const Backward &p, uint32_t id, float (&shared)[4])
{
    constexpr int ES = elem_size(DT), E = 16 / ES, N = 4;
    static_assert(16 * E >= FLASHLAYER_HEAD_MAX, "at most 16 granules");
    const int tile = id % p.key_tiles, problem = id / p.key_tiles, b = problem / p.Hk, g = problem - b * p.Hk;
    const int width = p.Dk, lanes = width <= 4 * E ? 4 : width <= 8 * E ? 8 : 16, step = 256 / lanes;
    const bool whole = width % E == 0;
    const int d = (threadIdx.x & (lanes - 1)) * E, end = (int)min((int64_t)p.keys(b), (int64_t)(tile + 1) * p.key_tile);
    const char *base = p.v + b * p.vb + g * p.vh;
    float most = 0.0f;
    for (int key0 = tile * p.key_tile + (int)threadIdx.x / lanes; key0 < end; key0 += step * N) {
        u32x4 w[N][1];
#pragma unroll
        for (int n = 0; n < N; ++n) {
            const char *row = base + (key0 + step * n) * p.vr;
            w[n][0] = u32x4{0, 0, 0, 0};
            if (key0 + step * n < end && d < width)
                w[n][0] = whole ? load16(row + d * ES) : load_granule_edge<DT>(row, d, width);
        }
#pragma unroll
        for (int n = 0; n < N; ++n) {
            float v[E], sq = 0.0f;
            elems_of<DT>(w[n], v);
#pragma unroll
            for (int i = 0; i < E; ++i) sq = __builtin_fmaf(v[i], v[i], sq);
            for (int o = 1; o < lanes; o *= 2) sq += __shfl_xor(sq, o);
            most = __builtin_fmaxf(most, sq);
        }
    }
#pragma unroll
    for (int o = 4; o < 64; o *= 2) most = __builtin_fmaxf(most, __shfl_xor(most, o));
    if ((threadIdx.x & 63) == 0) shared[threadIdx.x >> 6] = most;
    __syncthreads();
    if (threadIdx.x == 0)
        p.most_v[id] = sqrtf(__builtin_fmaxf(__builtin_fmaxf(shared[0], shared[1]), __builtin_fmaxf(shared[2], shared[3])));
}

// delta and (float16) |g| of a tile of 16 rows, 16 lanes to a row; and by the workgroups past the rows'
// float16's largest |v|.
template <int DT>
__global__ void __launch_bounds__(256) attend_rows(Backward p)
{
    constexpr int ES = elem_size(DT), E = 16 / ES;
    __shared__ float lds[3][4];
    const uint32_t id = block_index();
    if constexpr (DT == FLASHBEV_F16) {
        if (id >= p.row_blocks) {
            if (id - p.row_blocks < p.blocks_v) largest_values<DT>(p, id - p.row_blocks, lds[0]);
            return;
        }
    }
    if (id >= p.row_blocks) return;
    const int tile = id % p.row_tiles, problem = id / p.row_tiles;
    const int b = problem / p.Hk, g = problem - b * p.Hk;
    const int part = threadIdx.x & 15;
    float most_l = 0.0f, most_g = 0.0f, most_out = 0.0f;
    const int r = tile * kRowTile + (threadIdx.x >> 4);
    if (r < p.rows) {   // (whole groups of 16 lanes)
        int qi, qj;
        p.row(r, qi, qj);
        const int head = g * p.share + qj;
        const char *gr = p.g + b * p.ob + qi * p.orow + head * p.oh;
        const int64_t at = (((int64_t)b * p.Lq + qi) * p.H + head) * p.D;
        float delta = 0.0f, sq = 0.0f, sq_out = 0.0f;
        for (int d = part * E; d < p.D; d += 16 * E) {
            float vg[E], vo[E], vr[E];
            u32x4 w[1] = {load_granule_edge<DT>(gr, d, p.D)};
            elems_of<DT>(w, vg);
            w[0] = load_granule_edge<DT>(p.out + at * ES, d, p.D);
            elems_of<DT>(w, vo);
            if (p.rest) {
                w[0] = load_granule_edge<DT>(p.rest + at * ES, d, p.D);
                elems_of<DT>(w, vr);
            }
#pragma unroll
            for (int i = 0; i < E; ++i) {
                delta = __builtin_fmaf(vg[i], vo[i], delta);
                if (p.rest) delta = __builtin_fmaf(vg[i], vr[i], delta);
                if constexpr (DT == FLASHBEV_F16) {
                    sq = __builtin_fmaf(vg[i], vg[i], sq);
                    sq_out = __builtin_fmaf(vo[i], vo[i], sq_out);
                }
            }
        }
#pragma unroll
        for (int o = 1; o < 16; o *= 2) {
            delta += __shfl_xor(delta, o);
            sq += __shfl_xor(sq, o);
            sq_out += __shfl_xor(sq_out, o);
        }
        const float *st = p.stats + (((int64_t)b * p.H + head) * p.Lq + qi) * 2;
        RowData row;
        row.m = st[0];
        row.log2l = st[1] * kLog2;
        row.delta = delta;
        row.norm = sqrtf(sq);
        if (row.m == -__builtin_inff()) {
            row.m = 0.0f;
            row.log2l = __builtin_inff();
            row.delta = 0.0f;
        } else {
            const float inv = exp2_fast(-row.log2l);
            most_l = __builtin_fmaxf(most_l, inv);
            most_g = __builtin_fmaxf(most_g, row.norm * inv);
            most_out = __builtin_fmaxf(most_out, sqrtf(sq_out));
        }
        if (part == 0) {
            p.data[(int64_t)problem * p.rows + r] = row;
            p.lose[(int64_t)problem * p.padded + r] = __builtin_fmaf(row.m, kLog2, row.log2l);
            p.delta[(int64_t)problem * p.padded + r] = row.delta;
        }
    } else if (part == 0 && r < p.padded) {
        p.lose[(int64_t)problem * p.padded + r] = __builtin_inff();
        p.delta[(int64_t)problem * p.padded + r] = 0.0f;
    }
#pragma unroll
    for (int o = 16; o < 64; o *= 2) {
        most_l = __builtin_fmaxf(most_l, __shfl_xor(most_l, o));
        most_g = __builtin_fmaxf(most_g, __shfl_xor(most_g, o));
        most_out = __builtin_fmaxf(most_out, __shfl_xor(most_out, o));
    }
    if ((threadIdx.x & 63) == 0) {
        lds[0][threadIdx.x >> 6] = most_l;
        lds[1][threadIdx.x >> 6] = most_g;
        lds[2][threadIdx.x >> 6] = most_out;
    }
    __syncthreads();
    if (threadIdx.x < 3) {
        float v = lds[threadIdx.x][0];
        for (int w = 1; w < 4; ++w) v = __builtin_fmaxf(v, lds[threadIdx.x][w]);
        p.largest[3 * (int64_t)id + threadIdx.x] = v;
    }
}

// ---------------------------------------------------------------------------
// grad_q: 32 rows across to a wavefront, tiles of 64 keys
// ---------------------------------------------------------------------------
template <int DT, int DP>
struct ShapeQ {
    static constexpr int BQ = 128, BK = 64;
    using P = Panel<DT, DP, BK>;
    static constexpr int STAGE = 2 * P::BYTES, LDS = 2 * STAGE;
};

// Workgroups that are to run on a CU at once of the kernels with masks: two, whose wavefronts fill what one
// waits for, where 256 registers nearly do.  (They do up to heads of 64 16-bit channels; of 96 grad_k's and
// grad_v's kernel spills 41: the gradients at splits_of grad_q 50 -> 38 us, grad_k and grad_v 78 -> 61.  Heads of
// 128 take 368 and 447.)
constexpr int masked_waves(int bytes) { return bytes > 192 ? 1 : 2; }

template <int DT, int DP>
__global__ void __launch_bounds__(256, masked_waves(DP * elem_size(DT))) attend_grad_q(Backward p)
{
    using S = ShapeQ<DT, DP>;
    using P = typename S::P;
    constexpr int ES = elem_size(DT), DB = DP / 32;
    extern __shared__ __attribute__((aligned(16))) char lds[];

    uint32_t id = item_of(p);
    if (id >= p.blocks) return;
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tile = id % p.tiles;
    id /= p.tiles;
    const int split = id % p.splits;
    id /= p.splits;
    const int g = id % p.Hk, b = id / p.Hk;
    const int len = p.keys(b);
    const int all = (len + S::BK - 1) / S::BK, per = (all + p.splits - 1) / p.splits;
    const int t0 = split * per, t1 = min(all, t0 + per);

    const int r0 = tile * S::BQ + wave * 32, r = r0 + (lane & 31);
    const bool row_there = r < p.rows;
    int qi, qj;
    p.row(min(r, p.rows - 1), qi, qj);
    const int head = g * p.share + qj;
    u32x4 qf[P::CHUNKS], gf[P::CHUNKS];
    row_fragments<DT, DP>(qf, p.q + b * p.qb + qi * p.qr + head * p.qh, row_there, p.D, lane);
    row_fragments<DT, DP>(gf, p.g + b * p.ob + qi * p.orow + head * p.oh, row_there, p.D, lane);
    const char *mrow = p.mask + b * p.mb + head * p.mh + qi * p.mr;
    const RowData row = p.data[((int64_t)b * p.Hk + g) * p.rows + min(r, p.rows - 1)];
    // (weights are p l; an empty row's are exp(-inf - 0) = 0)
    const float inv = row_factor<DT>(p, row, (int64_t)b * p.Hk + g, lane), off = -row.delta * inv;
    const char *kbase = p.k + b * p.kb + g * p.kh, *vbase = p.v + b * p.vb + g * p.vh;
    f32x16 o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] = zeros16();

    typename P::Reader read;
    read.start(lane);
    typename P::Mover km, vm;
    km.start(tid, p.D, p.kr);
    vm.start(tid, p.D, p.vr);
    u32x4 kv[P::G], vv[P::G];
    km.clear(kv);
    vm.clear(vv);
    const bool copies = p.drops || p.D % P::E != 0;
    auto fetch = [&](int t) {
        if (copies) return;
        const int k0 = t * S::BK;
        km.load(kv, kbase + k0 * p.kr, p.kr, len - k0);
        vm.load(vv, vbase + k0 * p.vr, p.vr, len - k0);
    };
    auto put = [&](int t, char *lk, char *lv) {
        if (!copies) {
            km.store(kv, lk);
            vm.store(vv, lv);
            return;
        }
        const int k0 = t * S::BK;
        // (all rows' masks are the first one's where keys drop out)
        const auto there = [&](int i) { return !p.drops || mrow[k0 + i] != 0; };
        km.copy(lk, kbase + k0 * p.kr, p.kr, len - k0, p.D, there);
        vm.copy(lv, vbase + k0 * p.vr, p.vr, len - k0, p.D, there);
    };
    if (t0 < t1) fetch(t0);
    for (int t = t0; t < t1; ++t) {
        char *lk = lds + (t - t0 & 1) * S::STAGE, *lv = lk + P::BYTES;
        put(t, lk, lv);
        __syncthreads();
        if (t + 1 < t1) fetch(t + 1);
        if (r0 >= p.rows) continue;
#pragma unroll
        for (int n = 0; n < 2; ++n) {
            const int k0 = t * S::BK + n * 32;
            f32x16 x = zeros16(), y = zeros16();
            MaskBlock mask;
            mask.load_row(p, mrow, k0, h);
#pragma unroll
            for (int e = 0; e < P::CHUNKS; ++e) {
                mma<DT>(x, read.along(lk, n * 32, e), qf[e]);
                mma<DT>(y, read.along(lv, n * 32, e), gf[e]);
            }
            mask.apply_row(p, x);
            if (k0 + 32 > len) cut_keys(x, k0, h, len);
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const float w = exp2_fast((x[i] - row.m) * kLog2);
                x[i] = w * __builtin_fmaf(y[i], inv, off);
            }
#pragma unroll
            for (int u = 0; u < P::STEPS; ++u) {
                const u32x4 w = operand<DT>(x, u);
#pragma unroll
                for (int d = 0; d < DB; ++d) mma<DT>(o[d], read.across(lk, n * 32, u, d * 32), w);
            }
        }
    }
    if (!row_there) return;
    const float back = p.scale * exp2_fast(-row.log2l) / inv;
    const int64_t at = ((int64_t)b * p.Lq + qi) * p.H + head;
    const int64_t slot = ((int64_t)split * p.B * p.Lq * p.H + at) * DP;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            float v[8];
            columns_of(o[d], q, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= back;
            if (p.splits > 1) {
                store_elems<FLASHBEV_F32>(p.part + slot + d * 32 + 16 * q + 8 * h, v);
            } else {
                put8<DT>(p.gq + at * p.D * ES, d * 32 + 16 * q + 8 * h, p.D, v);
            }
        }
}

// ---------------------------------------------------------------------------
// grad_k and grad_v: 32 keys across to a wavefront, tiles of rows
// ---------------------------------------------------------------------------
// float16's factors (above) for rows r0 .. r1 - 1 of a problem: 2^up and 2^up times `more`, and times `key` of a
// lane's key.
template <int N>
__device__ __forceinline__ void factors(const Backward &p, int64_t problem, int r0, int r1, const u32x4 (&vf)[N],
                                        float (&shared)[3][4], float &up, float &more, float &key)
{
    const int tid = threadIdx.x, wave = tid >> 6;
    float most[3] = {0.0f, 0.0f, 0.0f};
    const float *at = p.largest + problem * p.row_tiles * 3;
    const int s1 = min(p.row_tiles, (r1 + kRowTile - 1) / kRowTile);
    for (int s = r0 / kRowTile + tid; s < s1; s += 256)
#pragma unroll
        for (int i = 0; i < 3; ++i) most[i] = __builtin_fmaxf(most[i], at[3 * s + i]);
#pragma unroll
    for (int i = 0; i < 3; ++i) {
#pragma unroll
        for (int o = 1; o < 64; o *= 2) most[i] = __builtin_fmaxf(most[i], __shfl_xor(most[i], o));
        if ((tid & 63) == 0) shared[i][wave] = most[i];
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 3; ++i)
        most[i] = __builtin_fmaxf(__builtin_fmaxf(shared[i][0], shared[i][1]), __builtin_fmaxf(shared[i][2], shared[i][3]));
    // (dS as in grad_q's kernel)
    const auto same = [](float v) {   // in all lanes
        return __builtin_bit_cast(float, __builtin_amdgcn_readfirstlane(__builtin_bit_cast(int, v)));
    };
    up = same(most[0] > 0.0f ? -__builtin_ceilf(log2_fast(most[0])) : 0.0f);
    const float down = most[1] > 0.0f && most[1] < __builtin_inff() ? -__builtin_ceilf(log2_fast(most[1])) : 0.0f;
    more = same(exp2_fast(within_range(down - 3.0f - up)));
    key = __builtin_ldexpf(1.0f, -spread_of_key(vf, most[2]));
}

// A key's gradients of a wavefront (both halves' channels), or its part of them.
template <int DT, int DP>
__device__ __forceinline__ void put_key(const Backward &p, int b, int g, int split, int key, bool key_there, float up,
                                        float more, const f32x16 (&ok)[DP / 32], const f32x16 (&ov)[DP / 32], int h)
{
    constexpr int ES = elem_size(DT), DB = DP / 32;
    if (key >= p.Lk) return;
    const float back_v = exp2_fast(-up), back_k = back_v * p.scale / more;
    const int64_t at = ((int64_t)b * p.Lk + key) * p.Hk + g, all_keys = (int64_t)p.B * p.Lk * p.Hk;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            float a[8], w[8];
            columns_of(ok[d], q, a);
            columns_of(ov[d], q, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) {   // (a key that is left out has sums of no meaning)
                a[i] = key_there ? a[i] * back_k : 0.0f;
                w[i] = key_there ? w[i] * back_v : 0.0f;
            }
            const int ch = d * 32 + 16 * q + 8 * h;
            if (p.splits > 1) {
                store_elems<FLASHBEV_F32>(p.part + (split * all_keys + at) * DP + ch, a);
                store_elems<FLASHBEV_F32>(p.part + ((p.splits + split) * all_keys + at) * DP + ch, w);
            } else {
                put8<DT>(p.gk + at * p.D * ES, ch, p.D, a);
                put8<DT>(p.gv + at * p.D * ES, ch, p.D, w);
            }
        }
}

template <int DT, int DP>
struct ShapeK {
    static constexpr int BK = 128;
    static constexpr int BR = DP * elem_size(DT) > 128 ? 32 : 64;
    using P = Panel<DT, DP, BR>;
    static constexpr int DATA = BR * 24;   // a row's mask (8 bytes), reference, exponent, delta
    static constexpr int STAGE = 2 * P::BYTES + DATA, LDS = 2 * STAGE;
};

// Scores, weights and products one after the other; other wavefronts fill the gaps.  900 x 40000 of
// 8 heads x 32 bf16 112 us, the vector units busy 69% of the time; with masks 3 x 777 x 1333 of 6
// heads x 72 half 61.
template <int DT, int DP, bool MASK>
__global__ void __launch_bounds__(256, masked_waves(DP * elem_size(DT))) attend_grad_kv(Backward p)
{
    using S = ShapeK<DT, DP>;
    using P = typename S::P;
    constexpr int DB = DP / 32;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ float shared[3][4];

    uint32_t id = item_of(p);
    if (id >= p.blocks) return;
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tile = id % p.tiles;
    id /= p.tiles;
    const int split = id % p.splits;
    id /= p.splits;
    const int g = id % p.Hk, b = id / p.Hk;
    const int64_t problem = (int64_t)b * p.Hk + g;
    const int len = p.keys(b);
    const int k0 = tile * S::BK + wave * 32, key = k0 + (lane & 31);
    const char *mbase = p.mask + b * p.mb + (int64_t)g * p.share * p.mh;
    const bool key_there = key < len && !(p.drops && mbase[key] == 0);

    const int all = tile * S::BK < len ? (p.rows + S::BR - 1) / S::BR : 0;
    const int per = (all + p.splits - 1) / p.splits;
    const int t0 = split * per, t1 = min(all, t0 + per);

    u32x4 kf[P::CHUNKS], vf[P::CHUNKS];
    const int64_t key_at = min(key, p.Lk - 1);
    row_fragments<DT, DP>(kf, p.k + b * p.kb + g * p.kh + key_at * p.kr, key_there, p.D, lane);
    row_fragments<DT, DP>(vf, p.v + b * p.vb + g * p.vh + key_at * p.vr, key_there, p.D, lane);
    const float c = (MASK ? 1.0f : p.scale) * kLog2;
    // the factors of p and dS: 2^up and 2^up `more`, which all keys have but for large values' own
    float up = 0.0f, all_keys = 1.0f, of_key = 1.0f;
    if constexpr (DT == FLASHBEV_F16) factors(p, problem, t0 * S::BR, t1 * S::BR, vf, shared, up, all_keys, of_key);
    // (large values are rare: without masks vector instructions are what bounds this, with them registers)
    const float more = MASK ? all_keys : all_keys * of_key;
    const bool large = DT == FLASHBEV_F16 && !MASK && __any(of_key != 1.0f);

    f32x16 ok[DB], ov[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) ok[d] = ov[d] = zeros16();

    typename P::Reader read;
    read.start(lane);
    // Rows on their way: row r is query r / share, head r % share.  A thread's places in a tile are
    // the same in every tile where tiles are whole queries.
    typename P::Mover mover;
    mover.start(tid, p.Dr, 0);
    const char *qbase = p.rq + b * p.rq_b + g * p.rq_g, *gbase = p.rg + b * p.rg_b + g * p.rg_g;
    const bool even = S::BR % p.rshare == 0, copies = MASK && p.D % P::E != 0;
    u32x4 qv[P::G], gv[P::G];
    mover.clear(qv);
    mover.clear(gv);
    uint32_t qoff[P::G], goff[P::G];
    RowData rd{};
    auto places = [&](int r0, int i0) {
#pragma unroll
        for (int i = 0; i < P::G; ++i) {
            int qi, qj;   // past the last row the last one again, whose weights are zeros
            p.part_of(min(r0 + mover.row + i * P::RP, p.rows - 1), qi, qj);
            qoff[i] = (uint32_t)(qi - i0) * (uint32_t)p.rq_r + (uint32_t)qj * (uint32_t)p.rq_h + mover.g * 16;
            goff[i] = (uint32_t)(qi - i0) * (uint32_t)p.rg_r + (uint32_t)qj * (uint32_t)p.rg_h + mover.g * 16;
        }
    };
    auto fetch = [&](int t) {
        const int r0 = t * S::BR;
        if (tid < S::BR && r0 + tid < p.rows) rd = p.data[problem * p.rows + r0 + tid];
        if (copies) return;
        const int i0 = r0 / p.rshare;
        if (t == t0 || !even || r0 + S::BR > p.rows) places(r0, i0);
        if (!mover.mine) return;
        const char *qt = qbase + i0 * p.rq_r, *gt = gbase + i0 * p.rg_r;
#pragma unroll
        for (int i = 0; i < P::G; ++i)
            if (mover.inside(i)) {
                qv[i] = load16(qt + qoff[i]);
                gv[i] = load16(gt + goff[i]);
            }
    };
    auto put = [&](int t, char *lq, char *lg, char *ld) {
        const int r0 = t * S::BR;
        if (tid < S::BR) {
            const bool there = r0 + tid < p.rows;
            if constexpr (MASK) {
                int qi, qj;
                p.row(there ? r0 + tid : 0, qi, qj);
                reinterpret_cast<int64_t *>(ld)[tid] = qi * p.mr + qj * p.mh;
            }
            float *f = reinterpret_cast<float *>(ld + 8 * S::BR);
            // rows past the last one weigh 2^-inf
            const float e = there ? rd.log2l - up : __builtin_inff();
            f[tid] = there ? rd.m : 0.0f;
            f[S::BR + tid] = MASK || !there ? e : __builtin_fmaf(rd.m, kLog2, e);
            f[2 * S::BR + tid] = there ? rd.delta * all_keys : 0.0f;
        }
        if (!copies) {
            mover.store(qv, lq);
            mover.store(gv, lg);
            return;
        }
        if (mover.row >= P::RP) return;
#pragma unroll 1
        for (int i = mover.row; i < S::BR; i += P::RP) {
            u32x4 a = {0, 0, 0, 0}, w = {0, 0, 0, 0};
            if (r0 + i < p.rows) {
                int qi, qj;
                p.row(r0 + i, qi, qj);
                a = P::granule(qbase + qi * p.rq_r + qj * p.rq_h, mover.g, p.D);
                w = P::granule(gbase + qi * p.rg_r + qj * p.rg_h, mover.g, p.D);
            }
            *reinterpret_cast<u32x4 *>(lq + P::place(i, mover.g)) = a;
            *reinterpret_cast<u32x4 *>(lg + P::place(i, mover.g)) = w;
        }
    };
    if (t0 < t1) fetch(t0);
    for (int t = t0; t < t1; ++t) {
        char *lq = lds + (t - t0 & 1) * S::STAGE, *lg = lq + P::BYTES, *ld = lg + P::BYTES;
        put(t, lq, lg, ld);
        __syncthreads();
        if (t + 1 < t1) fetch(t + 1);
        if (k0 >= len) continue;
#pragma unroll
        for (int n = 0; n < S::BR / 32; ++n) {
            f32x16 x = zeros16(), y = zeros16();
            [[maybe_unused]] MaskBlock mask;
            // (keys that are not there: the last one's, for sums of no meaning)
            if constexpr (MASK)
                mask.load_key(p, mbase, reinterpret_cast<const int64_t *>(ld) + n * 32 + 4 * h, min(key, p.Lk - 1));
#pragma unroll
            for (int e = 0; e < P::CHUNKS; ++e) {
                mma<DT>(x, read.along(lq, n * 32, e), kf[e]);
                mma<DT>(y, read.along(lg, n * 32, e), vf[e]);
            }
            if constexpr (MASK) mask.apply_key(p, x);
            const float *f = reinterpret_cast<const float *>(ld + 8 * S::BR) + n * 32 + 4 * h;
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const f32x4 e4 = *reinterpret_cast<const f32x4 *>(f + S::BR + 8 * k);
                f32x4 d4 = *reinterpret_cast<const f32x4 *>(f + 2 * S::BR + 8 * k);
                if (large) {
                    asm volatile("");   // (a branch, not selections)
#pragma unroll
                    for (int i = 0; i < 4; ++i) d4[i] *= of_key;
                }
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    float s = x[4 * k + i];
                    if constexpr (MASK) {
                        s = exp2_fast(__builtin_fmaf(s - f[8 * k + i], c, -e4[i]));
                    } else {
                        s = exp2_fast(__builtin_fmaf(s, c, -e4[i]));
                    }
                    x[4 * k + i] = s;
                    if constexpr (DT == FLASHBEV_F16 && MASK) s *= of_key;
                    y[4 * k + i] = s * __builtin_fmaf(y[4 * k + i], more, -d4[i]);
                }
            }
#pragma unroll
            for (int u = 0; u < P::STEPS; ++u) {
                const u32x4 wp = operand<DT>(x, u), ws = operand<DT>(y, u);
#pragma unroll
                for (int d = 0; d < DB; ++d) {
                    mma<DT>(ov[d], read.across(lg, n * 32, u, d * 32), wp);
                    mma<DT>(ok[d], read.across(lq, n * 32, u, d * 32), ws);
                }
            }
        }
    }
    put_key<DT, DP>(p, b, g, split, key, key_there, up, all_keys * of_key, ok, ov, h);
}

// ---------------------------------------------------------------------------
// without masks: loads that pass no registers, and one step's vector instructions among the
// products of the next and the last one, as the forward's attend_flow.  2 x 2048 x 4096 of 16
// heads x 128 on 4, bf16: grad_q 205 us (matrix units busy 56% of the time), grad_k and grad_v 300 (40%,
// one wavefront a SIMD); 900 x 40000 of 8 heads x 32: grad_q 98 (vector units busy 75%)
// ---------------------------------------------------------------------------
template <int DT, int DP>
struct FlowQ {
    static constexpr int TK = DP * elem_size(DT) <= 64 ? 128 : 64;
    static constexpr int SUBS = TK / 32;
    using T = Strip<DT, DP, TK>;
    static constexpr int LDS = 5 * T::BYTES;   // V of two tiles and K of three
};

// Wavefronts a SIMD, of heads of `bytes`.
constexpr int grad_q_waves(int bytes) { return bytes <= 64 ? 3 : bytes <= 256 ? 2 : 1; }

template <int DT, int DP, bool KEYS>
__global__ void __launch_bounds__(256, grad_q_waves(DP * elem_size(DT))) attend_grad_q_flow(Backward p)
{
    using F = FlowQ<DT, DP>;
    using T = typename F::T;
    constexpr int ES = elem_size(DT), DB = DP / 32, PAIRS = 8, E = T::E;
    extern __shared__ __attribute__((aligned(16))) char lds[];

    uint32_t id = item_of(p);
    if (id >= p.blocks) return;
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tile = id % p.tiles;
    id /= p.tiles;
    const int split = id % p.splits;
    id /= p.splits;
    const int g = id % p.Hk, b = id / p.Hk;
    const int len = p.keys(b);
    const int all = (len + F::TK - 1) / F::TK, per = (all + p.splits - 1) / p.splits;
    const int t0 = split * per, t1 = min(all, t0 + per), end = min(len, t1 * F::TK);

    const int r = tile * 128 + wave * 32 + (lane & 31);
    const bool row_there = r < p.rows;
    int qi, qj;
    p.row(min(r, p.rows - 1), qi, qj);
    const int head = g * p.share + qj;
    u32x4 qf[T::CHUNKS], gf[T::CHUNKS];
    row_fragments<DT, DP>(qf, p.q + b * p.qb + qi * p.qr + head * p.qh, row_there, p.D, lane);
    row_fragments<DT, DP>(gf, p.g + b * p.ob + qi * p.orow + head * p.oh, row_there, p.D, lane);
    const RowData row = p.data[((int64_t)b * p.Hk + g) * p.rows + min(r, p.rows - 1)];
    const float c = p.scale * kLog2, mc = row.m * kLog2;   // weights are p l
    const float inv = row_factor<DT>(p, row, (int64_t)b * p.Hk + g, lane), off = -row.delta * inv;

    f32x16 o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] = zeros16();

    typename T::Reader read;
    read.start(lane);
    typename T::Loader kl, vl;
    kl.start(wave, lane, p.Dk, p.kr);
    vl.start(wave, lane, p.Dk, p.vr);
    [[maybe_unused]] const uint32_t *words = p.words + b * p.words_b + g * p.words_g;
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds);
    const char *kbase = p.k + b * p.kb + g * p.kh, *vbase = p.v + b * p.vb + g * p.vh;
    const auto v_at = [&](int t) { return (t & 1) * T::BYTES; };
    const auto load = [&](int t, int k_at) {
        kl.load(kbase + t * F::TK * p.kr, len - t * F::TK, lds0 + k_at, wave);
        vl.load(vbase + t * F::TK * p.vr, len - t * F::TK, lds0 + v_at(t), wave);
    };

    // One step on scores x and products y of g with v: w, the packed dS; next_x and next_y of the 32
    // keys at lk and lv; and the product of the last step's dS with the 32 rows of k at lk0.
    const auto step = [&](auto first, f32x16 &x, f32x16 &y, f32x16 &next_x, f32x16 &next_y, u32x4(&w)[T::STEPS],
                          const u32x4(&last)[T::STEPS], const char *lk, const char *lv, const char *lk0, int key0) {
        constexpr bool FIRST = decltype(first)::value;
        constexpr int NS = T::CHUNKS, NP = T::STEPS * DB, N = 3 * NS, AHEAD = NS < 8 ? 3 : 2, Q = (PAIRS + NS - 1) / NS;
        static_assert(NS == NP, "as many products of each kind");
        const auto fragment = [&](int i) {
            return i % 3 == 0   ? read.along(lk, 0, i / 3)
                   : i % 3 == 1 ? read.along(lv, 0, i / 3)
                                : read.across(lk0, 0, i / 3 / DB, i / 3 % DB * 32);
        };
        if (key0 + 32 > end) cut_keys(x, key0, h, end);
        if constexpr (KEYS) {
            if (key0 < end) {
                const uint32_t word = words[key0 >> 5];
                if (word != 0xffffffffu) cut_word(x, word, h);
            }
        }
        float v[16];
        u32x4 f[AHEAD];
        next_x = zeros16();
        next_y = zeros16();
        asm volatile("" : "+v"(read.along_turn), "+v"(read.across_turn));
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            if (!FIRST || i % 3 != 2) f[i] = fragment(i);
#pragma unroll
        for (int i = 0; i < N + 6; ++i) {
            if (i < N) {
                if (i % 3 == 0) {
                    mma<DT>(next_x, f[i % AHEAD], qf[i / 3 % NS]);
                } else if (i % 3 == 1) {
                    mma<DT>(next_y, f[i % AHEAD], gf[i / 3 % NS]);
                } else if constexpr (!FIRST) {
                    mma<DT>(o[i / 3 % DB], f[i % AHEAD], last[i / 3 / DB % T::STEPS]);
                }
            }
            if (i + AHEAD < N && (!FIRST || (i + AHEAD) % 3 != 2)) f[i % AHEAD] = fragment(i + AHEAD);
            if (i % 3 == 0) {   // (few iterations: the compiler unrolls so much and no more)
#pragma unroll
                for (int n = 0; n < Q; ++n) {
                    if (const int j = (i / 3 - 2) * Q + n; j >= 0 && j < PAIRS) {
                        const int u = 2 * j / E, k = 2 * j % E;
                        v[2 * j] *= __builtin_fmaf(y[2 * j], inv, off);
                        v[2 * j + 1] *= __builtin_fmaf(y[2 * j + 1], inv, off);
                        if constexpr (DT == FLASHBEV_F32) {
                            w[u][k] = __builtin_bit_cast(uint32_t, v[2 * j]);
                            w[u][k + 1] = __builtin_bit_cast(uint32_t, v[2 * j + 1]);
                        } else {
                            w[u][k / 2] = pack2<DT>(v[2 * j], v[2 * j + 1]);
                        }
                    }
                    if (const int j = (i / 3 - 1) * Q + n; j >= 0 && j < PAIRS) {
                        v[2 * j] = exp2_fast(v[2 * j]);
                        v[2 * j + 1] = exp2_fast(v[2 * j + 1]);
                    }
                    if (const int j = i / 3 * Q + n; j < PAIRS) {
                        v[2 * j] = __builtin_fmaf(x[2 * j], c, -mc);
                        v[2 * j + 1] = __builtin_fmaf(x[2 * j + 1], c, -mc);
                    }
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    if (t0 < t1) {
        int k_now = 2 * T::BYTES, k_next = 3 * T::BYTES, k_free = 4 * T::BYTES;   // K of tiles t, t + 1, t + 2
        load(t0, k_now);
        if (t0 + 1 < t1) load(t0 + 1, k_next);
        meet();
        f32x16 x[2], y[2];
        u32x4 w[2][T::STEPS];
        x[0] = zeros16();
        y[0] = zeros16();
#pragma unroll
        for (int e = 0; e < T::CHUNKS; ++e) {
            mma<DT>(x[0], read.along(lds + k_now, 0, e), qf[e]);
            mma<DT>(y[0], read.along(lds + v_at(t0), 0, e), gf[e]);
        }
        step(std::true_type{}, x[0], y[0], x[1], y[1], w[0], w[1], lds + k_now + 32 * T::ROW,
             lds + v_at(t0) + 32 * T::ROW, lds, t0 * F::TK);
        for (int t = t0; t < t1; ++t) {
            // steps 1, 2, .. of the tile and step 0 of the next one, as the forward's
            const char *lk = lds + k_now, *lk2 = lds + k_next, *lv = lds + v_at(t), *lv2 = lds + v_at(t + 1);
#pragma unroll
            for (int s = 1; s <= F::SUBS; ++s) {
                if (s == F::SUBS - 1) {
                    meet();
                    if (t + 2 < t1) load(t + 2, k_free);
                }
                const int n = (s + 1) % F::SUBS * 32 * T::ROW;
                step(std::false_type{}, x[s & 1], y[s & 1], x[s + 1 & 1], y[s + 1 & 1], w[s & 1], w[s + 1 & 1],
                     (s + 1 < F::SUBS ? lk : lk2) + n, (s + 1 < F::SUBS ? lv : lv2) + n, lk + (s - 1) * 32 * T::ROW,
                     t * F::TK + s * 32);
            }
            const int turn = k_now;
            k_now = k_next;
            k_next = k_free;
            k_free = turn;
        }
    }
    if (!row_there) return;
    const float back = p.scale * exp2_fast(-row.log2l) / inv;
    const int64_t at = ((int64_t)b * p.Lq + qi) * p.H + head;
    const int64_t slot = ((int64_t)split * p.B * p.Lq * p.H + at) * DP;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            float v[8];
            columns_of(o[d], q, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= back;
            if (p.splits > 1) {
                store_elems<FLASHBEV_F32>(p.part + slot + d * 32 + 16 * q + 8 * h, v);
            } else {
                put8<DT>(p.gq + at * p.D * ES, d * 32 + 16 * q + 8 * h, p.D, v);
            }
        }
}

template <int DT, int DP>
struct FlowK {
    static constexpr int TR = DP * elem_size(DT) <= 64 ? 128 : 64;
    static constexpr int SUBS = TR / 32;
    using T = Strip<DT, DP, TR>;
    static constexpr int DATA = TR * 8;          // the rows' exponents and deltas
    static constexpr int STAGE = 2 * T::BYTES + DATA, LDS = 3 * STAGE;
    // Three stages of float32 heads of 128 channels are more than a CU's LDS: their gradients are
    // all taken by the kernels with masks.
    static constexpr bool ROOM = DP * elem_size(DT) < 512;
    static_assert(!ROOM || LDS <= 160 * 1024 - 64);
    // Heads of up to 32 16-bit channels have vector instructions for twice the products' time, and
    // four wavefronts a SIMD of attend_grad_kv do them faster than two of this kernel: 900 queries
    // x 40000 states 115 us and 131.
    static constexpr bool FITS = ROOM && DP * elem_size(DT) > 64;
};

constexpr int grad_kv_waves(int bytes) { return bytes <= 128 ? 2 : 1; }

template <int DT, int DP>
__global__ void __launch_bounds__(256, grad_kv_waves(DP * elem_size(DT))) attend_grad_kv_flow(Backward p)
{
    using F = FlowK<DT, DP>;
    using T = typename F::T;
    constexpr int DB = DP / 32, PAIRS = 8, E = T::E;
    extern __shared__ __attribute__((aligned(16))) char lds[];
    __shared__ float shared[3][4];

    uint32_t id = item_of(p);
    if (id >= p.blocks) return;
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int tile = id % p.tiles;
    id /= p.tiles;
    const int split = id % p.splits;
    id /= p.splits;
    const int g = id % p.Hk, b = id / p.Hk;
    const int64_t problem = (int64_t)b * p.Hk + g;
    const int len = p.keys(b);
    const int key = tile * 128 + wave * 32 + (lane & 31);
    const bool key_there =
        key < len && !(p.words && !(p.words[b * p.words_b + g * p.words_g + (key >> 5)] >> (key & 31) & 1));

    const int all = tile * 128 < len ? (p.rows + F::TR - 1) / F::TR : 0;
    const int per = (all + p.splits - 1) / p.splits;
    const int t0 = split * per, t1 = min(all, t0 + per);
    u32x4 kf[T::CHUNKS], vf[T::CHUNKS];
    const int64_t key_at = min(key, p.Lk - 1);
    row_fragments<DT, DP>(kf, p.k + b * p.kb + g * p.kh + key_at * p.kr, key_there, p.D, lane);
    row_fragments<DT, DP>(vf, p.v + b * p.vb + g * p.vh + key_at * p.vr, key_there, p.D, lane);
    const float c = p.scale * kLog2;
    float up = 0.0f, more = 1.0f;
    if constexpr (DT == FLASHBEV_F16) {
        float of_key;
        factors(p, problem, t0 * F::TR, t1 * F::TR, vf, shared, up, more, of_key);
        more *= of_key;
    }

    f32x16 ok[DB], ov[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) ok[d] = ov[d] = zeros16();

    typename T::Reader read;
    read.start(lane);
    typename T::RowLoader ql, gl;
    ql.start(wave, lane);
    gl.start(wave, lane);
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds);
    const char *qbase = p.rq + b * p.rq_b + g * p.rq_g, *gbase = p.rg + b * p.rg_b + g * p.rg_g;
    const float *lose = p.lose + problem * p.padded, *delta = p.delta + problem * p.padded;
    const bool even = F::TR % p.rshare == 0;   // a thread's places are the same in every tile
    const auto load = [&](int t, int stage) {
        const int r0 = t * F::TR, i0 = r0 / p.rshare;
        if (t == t0 || !even || r0 + F::TR > p.rows) {
            ql.places(p, r0, i0, p.rq_r, p.rq_h);
            gl.places(p, r0, i0, p.rg_r, p.rg_h);
        }
        ql.load(qbase + i0 * p.rq_r, p.Dr, lds0 + stage, wave);
        gl.load(gbase + i0 * p.rg_r, p.Dr, lds0 + stage + T::BYTES, wave);
        if (wave < 2 * F::TR / 64) {   // exponents, then deltas, 64 rows to an instruction
            const int part = wave * 64 % F::TR;
            word_to_lds((wave * 64 < F::TR ? lose : delta) + r0 + part + lane, lds0 + stage + 2 * T::BYTES + wave * 256);
        }
    };

    // One step on scores x and products y of the rows' g with v: wp and ws, the packed p and dS;
    // next_x and next_y of the 32 rows at lq and lg; and the products of the last step's p and dS
    // with the 32 rows at lq0 and lg0.
    const auto step = [&](auto first, f32x16 &x, f32x16 &y, f32x16 &next_x, f32x16 &next_y, u32x4(&wp)[T::STEPS],
                          u32x4(&ws)[T::STEPS], const u32x4(&last_p)[T::STEPS], const u32x4(&last_s)[T::STEPS],
                          const char *lq, const char *lg, const char *lq0, const char *lg0, const float *data) {
        constexpr bool FIRST = decltype(first)::value;
        constexpr int NS = T::CHUNKS, NP = T::STEPS * DB, N = 4 * NS, AHEAD = 4, Q = (PAIRS + NS - 1) / NS;
        static_assert(NS == NP, "as many products of each kind");
        const auto fragment = [&](int i) {
            return i % 4 == 0   ? read.along(lq, 0, i / 4)
                   : i % 4 == 1 ? read.along(lg, 0, i / 4)
                   : i % 4 == 2 ? read.across(lg0, 0, i / 4 / DB, i / 4 % DB * 32)
                                : read.across(lq0, 0, i / 4 / DB, i / 4 % DB * 32);
        };
        float v[16];
        u32x4 f[AHEAD];
        f32x4 e4[4], d4[4];
        next_x = zeros16();
        next_y = zeros16();
        asm volatile("" : "+v"(read.along_turn), "+v"(read.across_turn));
        const float *rows = data + 4 * h;
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            if (!FIRST || i % 4 < 2) f[i] = fragment(i);
#pragma unroll
        for (int k = 0; k < 4; ++k)
            if (2 * k / Q == 0) {
                e4[k] = *reinterpret_cast<const f32x4 *>(rows + 8 * k);
                d4[k] = *reinterpret_cast<const f32x4 *>(rows + F::TR + 8 * k);
            }
#pragma unroll
        for (int i = 0; i < N + 8; ++i) {
            if (i < N) {
                if (i % 4 == 0) {
                    mma<DT>(next_x, f[i % AHEAD], kf[i / 4 % NS]);
                } else if (i % 4 == 1) {
                    mma<DT>(next_y, f[i % AHEAD], vf[i / 4 % NS]);
                } else if constexpr (!FIRST) {
                    if (i % 4 == 2) {
                        mma<DT>(ov[i / 4 % DB], f[i % AHEAD], last_p[i / 4 / DB % T::STEPS]);
                    } else {
                        mma<DT>(ok[i / 4 % DB], f[i % AHEAD], last_s[i / 4 / DB % T::STEPS]);
                    }
                }
            }
            if (i + AHEAD < N && (!FIRST || (i + AHEAD) % 4 < 2)) f[i % AHEAD] = fragment(i + AHEAD);
            if (i % 4 == 0) {
#pragma unroll
                for (int k = 0; k < 4; ++k)   // the next pairs' rows
                    if (2 * k / Q > 0 && 2 * k / Q == i / 4 + 1) {
                        e4[k] = *reinterpret_cast<const f32x4 *>(rows + 8 * k);
                        d4[k] = *reinterpret_cast<const f32x4 *>(rows + F::TR + 8 * k);
                    }
            }
            if (i % 2 == 0) {
#pragma unroll
                for (int n = 0; n < Q; ++n) {
                    if (const int j = (i / 4 - 2) * Q + n; i % 4 == 0 && j >= 0 && j < PAIRS) {
                        const int u = 2 * j / E, at = 2 * j % E;
                        float s[2];
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            s[q] = v[2 * j + q] * (y[2 * j + q] - d4[j / 2][2 * j % 4 + q]);
                            if (DT == FLASHBEV_F16) s[q] *= more;
                        }
                        if constexpr (DT == FLASHBEV_F32) {
#pragma unroll
                            for (int q = 0; q < 2; ++q) {
                                wp[u][at + q] = __builtin_bit_cast(uint32_t, v[2 * j + q]);
                                ws[u][at + q] = __builtin_bit_cast(uint32_t, s[q]);
                            }
                        } else {
                            wp[u][at / 2] = pack2<DT>(v[2 * j], v[2 * j + 1]);
                            ws[u][at / 2] = pack2<DT>(s[0], s[1]);
                        }
                    }
                    if (const int j = (i / 4 - 1) * Q + n; i % 4 == 2 && j >= 0 && j < PAIRS) {
                        v[2 * j] = exp2_fast(v[2 * j]);
                        v[2 * j + 1] = exp2_fast(v[2 * j + 1]);
                    }
                    if (const int j = i / 4 * Q + n; i % 4 == 0 && j < PAIRS) {
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            const float e = e4[j / 2][2 * j % 4 + q];   // (a pair's rows in their four)
                            v[2 * j + q] = __builtin_fmaf(x[2 * j + q], c, DT == FLASHBEV_F16 ? up - e : -e);
                        }
                    }
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    };

    if (t0 < t1) {
        int now = 0, next = F::STAGE, free = 2 * F::STAGE;   // of tiles t, t + 1, t + 2
        load(t0, now);
        if (t0 + 1 < t1) load(t0 + 1, next);
        meet();
        f32x16 x[2], y[2];
        u32x4 wp[2][T::STEPS], ws[2][T::STEPS];
        x[0] = zeros16();
        y[0] = zeros16();
#pragma unroll
        for (int e = 0; e < T::CHUNKS; ++e) {
            mma<DT>(x[0], read.along(lds + now, 0, e), kf[e]);
            mma<DT>(y[0], read.along(lds + now + T::BYTES, 0, e), vf[e]);
        }
        constexpr int D0 = 2 * T::BYTES;
        step(std::true_type{}, x[0], y[0], x[1], y[1], wp[0], ws[0], wp[1], ws[1], lds + now + 32 * T::ROW,
             lds + now + T::BYTES + 32 * T::ROW, lds, lds, reinterpret_cast<const float *>(lds + now + D0));
        for (int t = t0; t < t1; ++t) {
            // Steps 1, 2, .. of the tile and step 0 of the next one (past the last tile for the last
            // step's products alone: its weights, of whatever lies there, are not used).
            const char *l0 = lds + now, *l1 = lds + next;
#pragma unroll
            for (int s = 1; s <= F::SUBS; ++s) {
                if (s == F::SUBS - 1) {
                    meet();
                    if (t + 2 < t1) load(t + 2, free);
                }
                const char *ln = (s + 1 < F::SUBS ? l0 : l1) + (s + 1) % F::SUBS * 32 * T::ROW;
                const char *lp = l0 + (s - 1) * 32 * T::ROW;
                const float *data = reinterpret_cast<const float *>((s < F::SUBS ? l0 : l1) + D0) + s % F::SUBS * 32;
                step(std::false_type{}, x[s & 1], y[s & 1], x[s + 1 & 1], y[s + 1 & 1], wp[s & 1], ws[s & 1],
                     wp[s + 1 & 1], ws[s + 1 & 1], ln, ln + T::BYTES, lp, lp + T::BYTES, data);
            }
            const int turn = now;
            now = next;
            next = free;
            free = turn;
        }
    }
    put_key<DT, DP>(p, b, g, split, key, key_there, up, more, ok, ov, h);
}

// The sums of the splits' rows [n][DP], four channels to a lane.
struct Sum {
    const float *part;
    char *out;
    int64_t n;
    int splits, D;
};

template <int DT, int DP>
__global__ void __launch_bounds__(256) attend_sum(Sum p)
{
    constexpr int LANES = DP / 4;
    const int64_t t = (int64_t)block_index() * 256 + threadIdx.x, at = t / LANES;
    const int d = (int)(t - at * LANES) * 4;
    if (at >= p.n || d >= p.D) return;
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 4
    for (int s = 0; s < p.splits; ++s) {
        const f32x4 v = *reinterpret_cast<const f32x4 *>(p.part + (s * p.n + at) * DP + d);
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += v[i];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (d + i < p.D) store_elem<DT>(p.out, at * p.D + d + i, sum[i]);
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
struct Plan {
    int dp, row_tiles, padded;
    bool any;      // masks that differ from row to row, and float32 heads of over 96 channels
    bool copies;   // k and v are copied first, and odd rows of q and g
    int q_tiles, q_splits;
    int k_tiles, k_splits;
};

Plan plan_of(const flashlayer_attention *a)
{
    Plan p{};
    const int64_t rows = (int64_t)a->Lq * (a->Hk ? a->H / a->Hk : 1), problems = (int64_t)a->B * a->Hk;
    p.dp = padded_head(a->D);
    p.any = pairs_of(a) || p.dp * elem_size(a->dtype) >= 512;
    p.copies = !p.any && copies_keys(a);
    p.padded = (int)((rows + 127) / 128 * 128);
    p.row_tiles = p.padded / kRowTile;
    p.q_tiles = (int)((rows + 127) / 128);
    p.k_tiles = (a->Lk + 127) / 128;
    // (steps of 64 keys, and of 64 rows)
    const int wide = p.dp * elem_size(a->dtype);
    p.q_splits = splits_of(problems * p.q_tiles, (a->Lk + 63) / 64, p.any ? masked_waves(wide) : grad_q_waves(wide));
    p.k_splits = splits_of(problems * p.k_tiles, (rows + 63) / 64, p.any ? masked_waves(wide) : grad_kv_waves(wide));
    return p;
}

uint64_t data_bytes(const flashlayer_attention *a)
{
    return align256((uint64_t)a->B * a->Lq * a->H * sizeof(RowData));
}

// the exponents and deltas for the kernel without masks
uint64_t rows_bytes(const flashlayer_attention *a, const Plan &p)
{
    return align256((uint64_t)a->B * a->Hk * p.padded * 4);
}

uint64_t copy_bytes(const flashlayer_attention *a, const Plan &p)
{
    if (!p.copies) return 0;
    return keys_copy_bytes(a) + (odd_of(a) ? 2 * rows_copy_bytes(a, (int64_t)a->Lq * share_of(a), a->Hk) : 0);
}

uint64_t largest_bytes(const flashlayer_attention *a, const Plan &p)
{
    return align256((uint64_t)a->B * a->Hk * p.row_tiles * 12);
}

// keys to a tile of largest |v|
int key_tile_of(const flashlayer_attention *a) { return std::max(128, ((a->Lk - 1) / kMostTiles + 16) / 16 * 16); }

int key_tiles_of(const flashlayer_attention *a)
{
    return a->dtype == FLASHBEV_F16 && a->Lk ? (a->Lk - 1) / key_tile_of(a) + 1 : 0;
}

uint64_t values_bytes(const flashlayer_attention *a)
{
    return align256((uint64_t)a->B * a->Hk * key_tiles_of(a) * 4);
}

uint64_t backward_bytes(const flashlayer_attention *a, bool want_q, bool want_kv)
{
    if (!a->B || !a->Lq || !a->H || !a->D) return 0;
    const Plan p = plan_of(a);
    uint64_t q = 0, kv = 0;   // one after the other in one place
    if (want_q && p.q_splits > 1)
        q = size_prod({(uint64_t)p.q_splits, (uint64_t)a->B * a->Lq * a->H, (uint64_t)p.dp, 4});
    if (want_kv && p.k_splits > 1)
        kv = size_prod({2, (uint64_t)p.k_splits, (uint64_t)a->B * a->Lk * a->Hk, (uint64_t)p.dp, 4});
    return copy_bytes(a, p) + data_bytes(a) + 2 * rows_bytes(a, p) + largest_bytes(a, p) + values_bytes(a) + align256(std::max(q, kv));
}

bool rows_to_lds(const Backward &p)
{
    return to_lds_reads(p.rq, {{p.B, p.rq_b}, {p.Hk, p.rq_g}, {p.Lq, p.rq_r}, {p.rshare, p.rq_h}}) &&
           to_lds_reads(p.rg, {{p.B, p.rg_b}, {p.Hk, p.rg_g}, {p.Lq, p.rg_r}, {p.rshare, p.rg_h}});
}

template <int DT, int DP>
int run(Backward &p, const Plan &plan, hipStream_t st)
{
    const uint64_t problems = (uint64_t)p.B * p.Hk;
    if (p.gq) {
        p.tiles = plan.q_tiles;
        p.splits = plan.q_splits;
        if (const int rc = deal(p, size_prod({problems, (uint64_t)p.tiles, (uint64_t)p.splits}))) return rc;
        const void *fn = (const void *)attend_grad_q<DT, DP>;
        size_t lds = ShapeQ<DT, DP>::LDS;
        if constexpr (FlowK<DT, DP>::ROOM) {
            if (!plan.any && keys_to_lds(p)) {
                fn = p.words ? (const void *)attend_grad_q_flow<DT, DP, true>
                             : (const void *)attend_grad_q_flow<DT, DP, false>;
                lds = FlowQ<DT, DP>::LDS;
            }
        }
        if (const int rc = launch_lds(fn, 8ull * p.per_xcd, p, lds, st)) return rc;
        if (p.splits > 1) {
            Sum s{p.part, p.gq, (int64_t)problems * p.rows, p.splits, p.D};
            const uint64_t lanes = (uint64_t)s.n * (DP / 4);
            if (const int rc = launch_rows((const void *)attend_sum<DT, DP>, (lanes + 255) / 256, 256, s, st)) return rc;
        }
    }
    if (!p.gk || !p.Lk) return FLASHBEV_OK;
    p.tiles = plan.k_tiles;
    p.splits = plan.k_splits;
    if (const int rc = deal(p, size_prod({problems, (uint64_t)p.tiles, (uint64_t)p.splits}))) return rc;
    const void *fn = (const void *)attend_grad_kv<DT, DP, true>;
    size_t lds = ShapeK<DT, DP>::LDS;
    if constexpr (DP * elem_size(DT) <= 64) {
        if (!plan.any) fn = (const void *)attend_grad_kv<DT, DP, false>;
    }
    if constexpr (FlowK<DT, DP>::FITS) {
        if (!plan.any && rows_to_lds(p)) {
            fn = (const void *)attend_grad_kv_flow<DT, DP>;
            lds = FlowK<DT, DP>::LDS;
        }
    }
    if (const int rc = launch_lds(fn, 8ull * p.per_xcd, p, lds, st)) return rc;
    if (p.splits <= 1) return FLASHBEV_OK;
    for (int half = 0; half < 2; ++half) {
        Sum s{p.part, half ? p.gv : p.gk, (int64_t)problems * p.Lk, p.splits, p.D};
        s.part += half * p.splits * s.n * DP;
        const uint64_t lanes = (uint64_t)s.n * (DP / 4);
        if (const int rc = launch_rows((const void *)attend_sum<DT, DP>, (lanes + 255) / 256, 256, s, st)) return rc;
    }
    return FLASHBEV_OK;
}

// grad_k and grad_v of no rows: zeros (a sum of no parts).
template <int DT>
int no_rows(const Backward &p, hipStream_t st)
{
    for (char *out : {p.gk, p.gv}) {
        Sum s{nullptr, out, (int64_t)p.B * p.Hk * p.Lk, 0, p.D};
        const uint64_t lanes = (uint64_t)s.n * (FLASHLAYER_HEAD_MAX / 4);
        if (const int rc = launch_rows((const void *)attend_sum<DT, FLASHLAYER_HEAD_MAX>, (lanes + 255) / 256, 256, s, st)) return rc;
    }
    return FLASHBEV_OK;
}

template <int DT>
int run_width(const flashlayer_attention *a, Backward &p, const Plan &plan, void *workspace, hipStream_t st)
{
    p.rq = p.q;
    p.rq_b = p.qb;
    p.rq_g = p.share * p.qh;
    p.rq_r = p.qr;
    p.rq_h = p.qh;
    p.rg = p.g;
    p.rg_b = p.ob;
    p.rg_g = p.share * p.oh;
    p.rg_r = p.orow;
    p.rg_h = p.oh;
    p.rshare = p.share;
    p.Dr = p.D;
    if (!p.rows) return no_rows<DT>(p, st);   // (and no mask: one of no rows has no address)
    if (plan.copies && a->Lk) {
        if (const int rc = copy_keys<DT>(a, p, static_cast<char *>(workspace), st)) return rc;
        if (odd_of(a) && p.gk) {
            Copy c{};
            const uint64_t each = rows_copy_bytes(a, p.rows, a->Hk);
            c.from[0] = p.q;
            c.from[1] = p.g;
            c.to[0] = static_cast<char *>(workspace) + keys_copy_bytes(a);
            c.to[1] = c.to[0] + each;
            c.batch[0] = p.qb;
            c.batch[1] = p.ob;
            c.row[0] = p.qr;
            c.row[1] = p.orow;
            c.head[0] = p.qh;
            c.head[1] = p.oh;
            c.group[0] = p.rq_g;
            c.group[1] = p.rg_g;
            c.heads = a->Hk;
            c.rows = p.rows;
            c.share = p.share;
            c.D = a->D;
            p.Dr = whole_head(a);
            c.granules = p.Dr * elem_size(DT) / 16;
            if (const int rc = copy_rows<DT>(c, a->B, st)) return rc;
            p.rq = c.to[0];
            p.rg = c.to[1];
            p.rq_r = p.rg_r = (int64_t)p.Dr * elem_size(DT);
            p.rq_h = p.rg_h = 0;
            p.rq_g = p.rg_g = p.rq_r * p.rows;
            p.rq_b = p.rg_b = p.rq_g * a->Hk;
            p.rshare = 1;
        }
    }
    const uint64_t tiles = size_prod({(uint64_t)p.B, (uint64_t)p.Hk, (uint64_t)plan.row_tiles});
    const uint64_t tiles_v = p.gq ? size_prod({(uint64_t)p.B, (uint64_t)p.Hk, (uint64_t)p.key_tiles}) : 0;   // (grad_q's)
    p.row_blocks = (uint32_t)tiles;   // (launch_rows refuses what does not fit)
    p.blocks_v = (uint32_t)tiles_v;
    if (const int rc = launch_rows((const void *)attend_rows<DT>, tiles + tiles_v, 256, p, st)) return rc;
    switch (plan.dp) {
    case 32: return run<DT, 32>(p, plan, st);
    case 64: return run<DT, 64>(p, plan, st);
    case 96: return run<DT, 96>(p, plan, st);
    default: return run<DT, 128>(p, plan, st);
    }
}

}  // namespace

extern "C" int flashlayer_attention_backward_workspace_size(const flashlayer_attention *args, int32_t want_q,
                                                            int32_t want_kv, uint64_t *bytes)
{
    if (!bytes) return FLASHBEV_ERR_NULLPTR;
    if (const int rc = check_attention(args)) return rc;
    *bytes = backward_bytes(args, want_q, want_kv);
    return FLASHBEV_OK;
}

extern "C" int flashlayer_attention_backward(const flashlayer_attention *args, const void *grad_out, const void *q,
                                             const void *k, const void *v, const void *mask,
                                             const int32_t *key_lengths, const void *out, const void *rest,
                                             const float *stats, void *grad_q, void *grad_k, void *grad_v,
                                             void *workspace, uint64_t workspace_bytes, void *stream)
{
    if (const int rc = check_attention(args)) return rc;
    const flashlayer_attention &a = *args;
    const int es = elem_size(a.dtype);
    const uint64_t rows = (uint64_t)a.B * a.Lq * a.H, keys = (uint64_t)a.B * a.Lk * a.Hk;
    // (a gradient without elements may be null)
    if (!a.B || !a.H || !a.D) return FLASHBEV_OK;
    if (keys && (!grad_k) != (!grad_v)) return FLASHBEV_ERR_NULLPTR;
    if (!(grad_q && rows) && !(grad_k && keys)) {
        return (!rows && grad_q) || (!keys && grad_k) || !rows || !keys ? FLASHBEV_OK : FLASHBEV_ERR_NULLPTR;
    }
    if ((rows && (!grad_out || !q || !out || !stats)) || (keys && (!k || !v))) return FLASHBEV_ERR_NULLPTR;
    if (a.mask && rows && keys && !mask) return FLASHBEV_ERR_NULLPTR;
    const int ms = a.mask == FLASHLAYER_MASK_BOOL ? 1 : a.mask == FLASHLAYER_MASK_ADD_F32 ? 4 : es;
    for (const void *t : {grad_out, q, k, v, out, rest, (const void *)grad_q, (const void *)grad_k, (const void *)grad_v})
        if (misaligned(t, es)) return FLASHBEV_ERR_ALIGN;
    if (misaligned(stats, 4) || misaligned(key_lengths, 4) || (a.mask && misaligned(mask, ms))) return FLASHBEV_ERR_ALIGN;
    const uint64_t need = backward_bytes(args, grad_q, grad_k);
    if (const int rc = check_scratch(workspace, workspace_bytes, need)) return rc;
    if (const int rc = check_overlaps(
            {{grad_q, rows * a.D * es}, {grad_k, keys * a.D * es}, {grad_v, keys * a.D * es}, {workspace, need}},
            {{grad_out, span4(a.B, a.o_batch, a.Lq, a.o_row, a.H, a.o_head, a.D, es)},
             {q, span4(a.B, a.q_batch, a.Lq, a.q_row, a.H, a.q_head, a.D, es)},
             {k, span4(a.B, a.k_batch, a.Lk, a.k_row, a.Hk, a.k_head, a.D, es)},
             {v, span4(a.B, a.v_batch, a.Lk, a.v_row, a.Hk, a.v_head, a.D, es)},
             {a.mask ? mask : nullptr, span4(a.B, a.mask_batch, a.H, a.mask_head, a.Lq, a.mask_row, a.Lk, ms)},
             {key_lengths, (uint64_t)a.B * 4},
             {out, rows * a.D * es},
             {rest, rows * a.D * es},
             {stats, rows * 8}}))
        return rc;
    const Plan plan = plan_of(args);
    Backward p{};
    static_cast<Attend &>(p) = attend_of(args);
    p.q = static_cast<const char *>(q);
    p.k = static_cast<const char *>(k);
    p.v = static_cast<const char *>(v);
    p.g = static_cast<const char *>(grad_out);
    p.mask = static_cast<const char *>(mask);
    p.lengths = key_lengths;
    p.out = static_cast<const char *>(out);
    p.rest = static_cast<const char *>(rest);
    p.stats = stats;
    p.gq = static_cast<char *>(grad_q);
    p.gk = static_cast<char *>(grad_k);
    p.gv = static_cast<char *>(grad_v);
    p.row_tiles = plan.row_tiles;
    p.padded = plan.padded;
    char *ws = static_cast<char *>(workspace) + copy_bytes(args, plan);
    p.data = reinterpret_cast<RowData *>(ws);
    ws += data_bytes(args);
    p.lose = reinterpret_cast<float *>(ws);
    ws += rows_bytes(args, plan);
    p.delta = reinterpret_cast<float *>(ws);
    ws += rows_bytes(args, plan);
    p.largest = reinterpret_cast<float *>(ws);
    ws += largest_bytes(args, plan);
    p.most_v = reinterpret_cast<float *>(ws);
    p.key_tiles = key_tiles_of(args);
    p.key_tile = key_tile_of(args);
    p.part = reinterpret_cast<float *>(ws + values_bytes(args));
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (a.dtype == FLASHBEV_F32) return run_width<FLASHBEV_F32>(args, p, plan, workspace, st);
    return a.dtype == FLASHBEV_F16 ? run_width<FLASHBEV_F16>(args, p, plan, workspace, st) : run_width<FLASHBEV_BF16>(args, p, plan, workspace, st);
}
