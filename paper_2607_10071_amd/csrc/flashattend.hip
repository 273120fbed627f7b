// Attention of queries to the states of an encoder of another length, for AMD MI355X (gfx950).
// C ABI: include/block/flashlayer.h; what the backward shares: flashattend.h.
//
//   out = softmax(scale q k^T + mask) v
//
// One pass over the keys.  A row keeps a reference m of its scores, the sum l of exp(s - m) and
// the sums of exp(s - m) v; when a score passes m by more than a few powers of two, all three
// move to the new maximum.  Nothing of the scores is stored.
#include <hip/hip_runtime.h>
#include <math.h>
#include <stdint.h>

#include <type_traits>

#include "flashattend.h"

namespace {

struct Forward : Attend {
    char *rest;          // null: not wanted
    float *stats;        // null: not wanted
    float *part;         // splits > 1: [splits][B Hk rows][DP] sums, then [..][2] m and l
    float *part_ml;
    int any;             // the kernels with masks: scores are scaled, references are theirs
};

// How large weights exp(s - m) may become before the reference m moves: within float16's range
// with room for the backward's factors, and above the 16 that a lane's share of 32 equal scores
// adds up to, where sums are looked at.
template <int DT>
constexpr float kLargest = DT == FLASHBEV_F16 ? 64.0f : 256.0f;

// l and the weights' sums, of two packed weights: the sum takes them as the product with v does,
// rounded, so that the result is a mean of v's rows with weights that add up to one.
template <int DT>
__device__ __forceinline__ float add_weights(float l, uint32_t two)
{
    if constexpr (DT == FLASHBEV_F16) {
        typedef _Float16 h2 __attribute__((ext_vector_type(2)));
        return __builtin_amdgcn_fdot2(__builtin_bit_cast(h2, two), h2{(_Float16)1.0f, (_Float16)1.0f}, l, false);
    } else {
        typedef __bf16 b2 __attribute__((ext_vector_type(2)));
        return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(b2, two), b2{(__bf16)1.0f, (__bf16)1.0f}, l, false);
    }
}

// A row's result of a wavefront (both halves' channels), or its part of one.
template <int DT, int DP, bool MASK>
__device__ __forceinline__ void put_row(const Forward &p, int b, int g, int split, int r, int qi, int head, float m,
                                        float l, const f32x16 (&o)[DP / 32], int h)
{
    constexpr int ES = elem_size(DT), DB = DP / 32;
    if (r >= p.rows) return;

    if (p.splits > 1) {
        const int64_t at = ((int64_t)split * p.B * p.Hk + (int64_t)b * p.Hk + g) * p.rows + r;
        float *part = p.part + at * DP;
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                float v[8];
                columns_of(o[d], q, v);
                store_elems<FLASHBEV_F32>(part + d * 32 + 16 * q + 8 * h, v);
            }
        if (!h) {
            p.part_ml[2 * at] = m;
            p.part_ml[2 * at + 1] = l;
        }
        return;
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;   // (a row that sees nothing)
    char *out = p.o + b * p.ob + qi * p.orow + head * p.oh;
    char *rest = p.rest ? p.rest + (((int64_t)b * p.Lq + qi) * p.H + head) * p.D * ES : nullptr;
#pragma unroll
    for (int d = 0; d < DB; ++d)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
            float v[8];
            columns_of(o[d], q, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] *= inv;
            put8<DT>(out, d * 32 + 16 * q + 8 * h, p.D, v);
            if (rest) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] -= rounded<DT>(v[i]);
                put8<DT>(rest, d * 32 + 16 * q + 8 * h, p.D, v);
            }
        }
    if (p.stats && !h) {
        float *st = p.stats + (((int64_t)b * p.H + head) * p.Lq + qi) * 2;
        st[0] = MASK ? m : m * p.scale;
        st[1] = l == 0.0f ? 0.0f : log2_fast(l) * kLn2;
    }
}

// WQ = 4: a wavefront has 32 rows, the four of them share tiles of 64 keys.  WQ = 1: the
// wavefronts share 32 rows and take 32 keys each of tiles of 128; their results are joined.
// Few rows read each key once and little else: tokens of 8 sequences, 32 heads on 8 x 128 bf16, caches of
// 3712 to 8192: 195 MB read in 45 us, 4.3 TB/s.  Each XCD has one of the sequences there, and the longest one's 34 MB
// take as long.  With masks a wavefront's products, masks and exponentials wait for each
// other: 3 x 777 queries by 1333 keys of 6 heads x 72 half with a bias 36 us, the matrix units
// busy 10% of the time, the vector units 29%.
template <int DT, int DP, int WQ>
struct Shape {
    static constexpr int BQ = 32 * WQ;
    static constexpr int BK = WQ == 4 ? 64 : 128;
    static constexpr int NB = WQ == 4 ? 2 : 1;         // blocks of 32 keys a wavefront has of a tile
    static constexpr int STAGES = WQ == 4 ? 2 : 1;
    using P = Panel<DT, DP, BK>;
    static constexpr int STAGE = 2 * P::BYTES;
    static constexpr int JOIN = WQ == 4 ? 0 : 2 * DP * 32 * 4 + 1024;
    static constexpr int LDS = STAGES * STAGE > JOIN ? STAGES * STAGE : JOIN;
};

// MASK: with a mask or rows that end inside a granule (that code in kernels of its own: it takes
// registers).  Wide float32 heads take one workgroup's registers of a CU.
template <int DT, int DP, int WQ, bool MASK>
__global__ void __launch_bounds__(256, DT == FLASHBEV_F32 && DP > 64 ? 1 : 2) attend(Forward p)
{
    using S = Shape<DT, DP, WQ>;
    using P = typename S::P;
    constexpr int NB = S::NB, DB = DP / 32;
    extern __shared__ __attribute__((aligned(16))) char lds[];

    uint32_t id = item_of(p);
    if (id >= p.blocks) return;
    const int tid = threadIdx.x, lane = tid & 63, h = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    int tile = 0, split, g, b;
    if (p.tiles == 1) {   // heads next to each other, whose keys' rows share cache lines
        g = id % p.Hk;
        id /= p.Hk;
        split = id % p.splits;
        b = id / p.splits;
    } else {
        tile = id % p.tiles;
        id /= p.tiles;
        split = id % p.splits;
        id /= p.splits;
        g = id % p.Hk;
        b = id / p.Hk;
    }
    const int len = p.keys(b);
    const int all = (len + S::BK - 1) / S::BK, per = (all + p.splits - 1) / p.splits;
    const int t0 = split * per, t1 = min(all, t0 + per);

    const int r0 = tile * S::BQ + (WQ == 4 ? wave * 32 : 0), r = r0 + (lane & 31);
    const bool row_there = r < p.rows;
    int qi, qj;
    p.row(min(r, p.rows - 1), qi, qj);
    const int head = g * p.share + qj;
    u32x4 qf[P::CHUNKS];
    row_fragments<DT, DP>(qf, p.q + b * p.qb + qi * p.qr + head * p.qh, row_there, p.D, lane);
    const char *mrow = p.mask + b * p.mb + head * p.mh + qi * p.mr;
    const char *kbase = p.k + b * p.kb + g * p.kh, *vbase = p.v + b * p.vb + g * p.vh;
    const float c = (MASK ? 1.0f : p.scale) * kLog2;   // of x, to powers of two

    f32x16 o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] = zeros16();
    float m = -__builtin_inff(), l = 0.0f;

    typename P::Reader read;
    read.start(lane);
    typename P::Mover km, vm;
    km.start(tid, p.D, p.kr);
    vm.start(tid, p.D, p.vr);
    u32x4 kv[P::G], vv[P::G];
    km.clear(kv);
    vm.clear(vv);
    const bool copies = MASK && (p.drops || p.D % P::E != 0);
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
        char *lk = lds + (S::STAGES > 1 ? (t - t0 & 1) * S::STAGE : 0), *lv = lk + P::BYTES;
        if (S::STAGES == 1 && t > t0) __syncthreads();
        put(t, lk, lv);
        __syncthreads();
        if (t + 1 < t1) fetch(t + 1);
        if (WQ == 4 && r0 >= p.rows) continue;
        const int b0 = WQ == 4 ? 0 : wave * 32;   // the wavefront's first key of the tile
        const int k0 = t * S::BK + b0;
        lk += b0 * P::STRIDE;
        lv += b0 * P::STRIDE;
        f32x16 x[NB];
        [[maybe_unused]] MaskBlock mask[NB];
        if constexpr (MASK) {
#pragma unroll
            for (int n = 0; n < NB; ++n) mask[n].load_row(p, mrow, k0 + n * 32, h);
        }
#pragma unroll
        for (int n = 0; n < NB; ++n) {
            x[n] = zeros16();
#pragma unroll
            for (int e = 0; e < P::CHUNKS; ++e) mma<DT>(x[n], read.along(lk, n * 32, e), qf[e]);
        }
        if constexpr (MASK) {
#pragma unroll
            for (int n = 0; n < NB; ++n) mask[n].apply_row(p, x[n]);
        }
        if (k0 + NB * 32 > len) {
#pragma unroll
            for (int n = 0; n < NB; ++n) cut_keys(x[n], k0 + n * 32, h, len);
        }
        float top = x[0][0];
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) top = __builtin_fmaxf(top, x[n][i]);
        top = both_max(top);
        if (__any(exp2_fast((top - m) * c) > kLargest<DT>)) {   // (-inf - -inf is no number, and not above)
            const float to = __builtin_fmaxf(m, top);
            const float f = to == -__builtin_inff() ? 1.0f : exp2_fast((m - to) * c);
            m = to;
            l *= f;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= f;
        }
        const float ref = m == -__builtin_inff() ? 0.0f : m;
        if constexpr (MASK) {
            // the difference first: x and m may be the type's lowest values, whose products
            // with log2(e) are infinite
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) x[n][i] = exp2_fast((x[n][i] - ref) * c);
        } else {
            const float mc = ref * c;
#pragma unroll
            for (int n = 0; n < NB; ++n)
#pragma unroll
                for (int i = 0; i < 16; ++i) x[n][i] = exp2_fast(__builtin_fmaf(x[n][i], c, -mc));
        }
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int u = 0; u < P::STEPS; ++u) {
                const u32x4 w = operand<DT>(x[n], u);
                if constexpr (DT == FLASHBEV_F32) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) l += x[n][4 * u + i];
                } else {
#pragma unroll
                    for (int i = 0; i < 4; ++i) l = add_weights<DT>(l, w[i]);
                }
#pragma unroll
                for (int d = 0; d < DB; ++d) mma<DT>(o[d], read.across(lv, n * 32, u, d * 32), w);
            }
    }
    l = both_sum(l);

    if constexpr (WQ == 1) {
        // the wavefronts' results, at the largest of their references
        float *ml = reinterpret_cast<float *>(lds), *area = ml + 256;
        __syncthreads();
        if (lane < 32) {
            ml[wave * 32 + lane] = m;
            ml[128 + wave * 32 + lane] = l;
        }
        __syncthreads();
        float to = -__builtin_inff(), sum = 0.0f;
#pragma unroll
        for (int w = 0; w < 4; ++w) to = __builtin_fmaxf(to, ml[w * 32 + (lane & 31)]);
        const auto factor = [&](float from) {
            return from == -__builtin_inff() ? 0.0f : exp2_fast((from - to) * c);
        };
#pragma unroll
        for (int w = 0; w < 4; ++w)
            sum += ml[128 + w * 32 + (lane & 31)] * factor(ml[w * 32 + (lane & 31)]);
        const float f = factor(m);
#pragma unroll
        for (int d = 0; d < DB; ++d)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] *= f;
        m = to;
        l = sum;
#pragma unroll
        for (int half = 2; half > 0; half /= 2) {
            if (wave >= half && wave < 2 * half) {
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i)
                        area[(((wave - half) * DB + d) * 16 + i) * 64 + lane] = o[d][i];
            }
            __syncthreads();
            if (wave < half) {
#pragma unroll
                for (int d = 0; d < DB; ++d)
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[d][i] += area[((wave * DB + d) * 16 + i) * 64 + lane];
            }
            __syncthreads();
        }
        if (wave) return;
    }
    put_row<DT, DP, MASK>(p, b, g, split, r, qi, head, m, l, o, h);
}

// Without masks that differ from row to row: four wavefronts of 32 rows each share tiles of TK keys,
// which go from memory to LDS without passing registers, and take them 32 keys at a time.  In one
// step a wavefront forms the next 32 keys' scores, this 32's weights and the product of the last 32's with v: matrix
// and vector instructions that do not wait for each other, in turn.  (Scores, then weights, then
// the product: 2048 queries of 32 heads x 4096 keys x 128 bf16 165 us.)
//
// Heads of 32 are bound by vector instructions: by the counters a step has 16 exponentials of 8 clocks, 46
// others of 4 and the issue of 4 products, 330 clocks of the 396 that it takes (16 of the others scale scores, 8
// round weights, 8 sum them), and the products 128.  40000 queries x 8700 keys of 8 heads, bf16, 519 us at some 2.0
// GHz, the vector units busy 83% of the time, the matrix units 32%. Wide heads by both and what they
// wait for each other: the case above 150 us, 49% each, 920 TFLOP/s.
template <int DT, int DP>
struct Flow {
    static constexpr int TK = DP * elem_size(DT) <= 64 ? 128 : 64;
    static constexpr int SUBS = TK / 32;
    using T = Strip<DT, DP, TK>;
    // K of two tiles and V of three: a tile's last product is taken with the next one's first step
    static constexpr int LDS = 5 * T::BYTES;
};

// Wavefronts a SIMD that the registers are to leave room for.
constexpr int flow_waves(int dt, int dp)
{
    return dp * elem_size(dt) <= 64 ? 4 : dp * elem_size(dt) < 512 ? 2 : 1;
}

// KEYS: some keys are left out, by their bits.
template <int DT, int DP, bool KEYS>
__global__ void __launch_bounds__(256, flow_waves(DT, DP)) attend_flow(Forward p)
{
    using F = Flow<DT, DP>;
    using T = typename F::T;
    constexpr int DB = DP / 32, PAIRS = 8, E = T::E;
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
    int qi, qj;
    p.row(min(r, p.rows - 1), qi, qj);
    const int head = g * p.share + qj;
    u32x4 qf[T::CHUNKS];
    row_fragments<DT, DP>(qf, p.q + b * p.qb + qi * p.qr + head * p.qh, r < p.rows, p.D, lane);
    const float c = p.scale * kLog2;   // of scores, to powers of two

    f32x16 o[DB];
#pragma unroll
    for (int d = 0; d < DB; ++d) o[d] = zeros16();
    float m = -__builtin_inff(), l = 0.0f;

    typename T::Reader read;
    read.start(lane);
    typename T::Loader kl, vl;
    kl.start(wave, lane, p.Dk, p.kr);
    vl.start(wave, lane, p.Dk, p.vr);
    [[maybe_unused]] const uint32_t *words = p.words + b * p.words_b + g * p.words_g;
    const uint32_t lds0 = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)(__attribute__((address_space(3))) char *)lds);
    const char *kbase = p.k + b * p.kb + g * p.kh, *vbase = p.v + b * p.vb + g * p.vh;
    // K of tile t lies at k_at(t); V's places turn by one a tile
    const auto k_at = [&](int t) { return (t & 1) * T::BYTES; };
    const auto load = [&](int t, int v_at) {
        kl.load(kbase + t * F::TK * p.kr, len - t * F::TK, lds0 + k_at(t), wave);
        vl.load(vbase + t * F::TK * p.vr, len - t * F::TK, lds0 + v_at, wave);
    };

    // Weights 2 j and 2 j + 1 of a step: their exponents, their powers, and the packed word, which
    // the lane's sum takes as it is.
    const auto exponents = [&](const f32x16 &x, float(&v)[16], int j, float mc) {
#pragma unroll
        for (int i = 2 * j; i < 2 * j + 2; ++i) v[i] = __builtin_fmaf(x[i], c, -mc);
    };
    const auto powers = [&](float(&v)[16], int j) {
#pragma unroll
        for (int i = 2 * j; i < 2 * j + 2; ++i) v[i] = exp2_fast(v[i]);
    };
    const auto packed = [&](const float(&v)[16], u32x4(&w)[T::STEPS], float &sum, int j) {
        const int u = 2 * j / E, i = 2 * j % E;
        if constexpr (DT == FLASHBEV_F32) {
            w[u][i] = __builtin_bit_cast(uint32_t, v[2 * j]);
            w[u][i + 1] = __builtin_bit_cast(uint32_t, v[2 * j + 1]);
            sum += v[2 * j];
            sum += v[2 * j + 1];
        } else {
            w[u][i / 2] = pack2<DT>(v[2 * j], v[2 * j + 1]);
            sum = add_weights<DT>(sum, w[u][i / 2]);
        }
    };

    // One step on scores x and their weights w: `next` scores of the 32 keys at lk, and the
    // product of the last step's weights with the 32 rows of v at lv (FIRST: there are none).
    const auto step = [&](auto first, f32x16 &x, f32x16 &next, u32x4(&w)[T::STEPS], const u32x4(&last)[T::STEPS],
                          const char *lk, const char *lv, int key0) {
        constexpr bool FIRST = decltype(first)::value;
        // products: scores' at even places, v's at odd ones
        constexpr int NS = T::CHUNKS, NP = FIRST ? 0 : T::STEPS * DB, N = 2 * (NS > NP ? NS : NP);
        constexpr int AHEAD = 4, Q = (PAIRS * 2 + N - 1) / N;   // pairs of weights to two products
        const auto is = [](int i) { return i % 2 == 0 ? i / 2 < NS : i / 2 < NP; };
        const auto fragment = [&](int i) {
            return i % 2 == 0 ? read.along(lk, 0, i / 2) : read.across(lv, 0, i / 2 / DB, i / 2 % DB * 32);
        };
        if (key0 + 32 > end) cut_keys(x, key0, h, end);
        if constexpr (KEYS) {
            if (key0 < end) {
                const uint32_t word = words[key0 >> 5];
                if (word != 0xffffffffu) cut_word(x, word, h);
            }
        }
        const float mc = m * c;
        float v[16], sum = 0.0f;
        u32x4 f[AHEAD];
        next = zeros16();
        // (places are formed again for every step: kept over the loop they spilled)
        asm volatile("" : "+v"(read.along_turn), "+v"(read.across_turn));
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            if (is(i)) f[i] = fragment(i);
#pragma unroll
        for (int i = 0; i < N + 4; ++i) {
            if (i < N && is(i)) {
                if (i % 2 == 0) {
                    mma<DT>(next, f[i % AHEAD], qf[i / 2 % NS]);
                } else if constexpr (!FIRST) {
                    mma<DT>(o[i / 2 % DB], f[i % AHEAD], last[i / 2 / DB % T::STEPS]);
                }
            }
            if (i + AHEAD < N && is(i + AHEAD)) f[i % AHEAD] = fragment(i + AHEAD);
            if (i % 2 == 0) {
#pragma unroll
                for (int n = 0; n < Q; ++n) {
                    if (const int j = (i / 2 - 2) * Q + n; j >= 0 && j < PAIRS) packed(v, w, sum, j);
                    if (const int j = (i / 2 - 1) * Q + n; j >= 0 && j < PAIRS) powers(v, j);
                    if (const int j = i / 2 * Q + n; j < PAIRS) exponents(x, v, j, mc);
                }
            }
            __builtin_amdgcn_sched_barrier(0);
        }
        // A reference that is too low shows in the sum of its weights; so does one that is not set
        // yet, -inf, in weights that are infinite or no numbers.  (No maximum is taken of the
        // other steps' scores.)
        if (__any(!(sum <= kLargest<DT>))) {
            asm volatile("");
            float top = x[0];
#pragma unroll
            for (int i = 0; i < 16; ++i) top = __builtin_fmaxf(top, x[i]);
            const float to = __builtin_fmaxf(m, both_max(top));
            const float by = m == -__builtin_inff() ? 0.0f : exp2_fast((m - to) * c);
            // (scores that are all -inf leave the reference unset, and weights of 0)
            const float at = (to == -__builtin_inff() ? 0.0f : to) * c;
            m = to;
            l *= by;
#pragma unroll
            for (int d = 0; d < DB; ++d)
#pragma unroll
                for (int i = 0; i < 16; ++i) o[d][i] *= by;
            sum = 0.0f;
#pragma unroll
            for (int j = 0; j < PAIRS; ++j) {
                exponents(x, v, j, at);
                powers(v, j);
                packed(v, w, sum, j);
            }
        }
        l += sum;
    };

    if (t0 < t1) {
        int v_now = 2 * T::BYTES, v_next = 3 * T::BYTES, v_free = 4 * T::BYTES;   // V of tiles t, t + 1, t + 2
        load(t0, v_now);
        if (t0 + 1 < t1) load(t0 + 1, v_next);
        meet();
        f32x16 x[2];
        u32x4 w[2][T::STEPS];
        x[0] = zeros16();
#pragma unroll
        for (int e = 0; e < T::CHUNKS; ++e) mma<DT>(x[0], read.along(lds + k_at(t0), 0, e), qf[e]);
        step(std::true_type{}, x[0], x[1], w[0], w[1], lds + k_at(t0) + 32 * T::ROW, lds, t0 * F::TK);
        for (int t = t0; t < t1; ++t) {
            // Steps 1, 2, .. of the tile and step 0 of the next one (past the last tile it only takes
            // the last step's product: its scores, of whatever lies there, are all cut).
            const char *lk = lds + k_at(t), *lk2 = lds + k_at(t + 1), *lv = lds + v_now;
#pragma unroll
            for (int s = 1; s <= F::SUBS; ++s) {
                if (s == F::SUBS - 1) {
                    // the next tile is there; K's place of this one is free, and a third one of V's
                    meet();
                    if (t + 2 < t1) load(t + 2, v_free);
                }
                const char *k_next = s + 1 < F::SUBS ? lk + (s + 1) * 32 * T::ROW : lk2 + (s + 1 - F::SUBS) * 32 * T::ROW;
                step(std::false_type{}, x[s & 1], x[s + 1 & 1], w[s & 1], w[s + 1 & 1], k_next,
                     lv + (s - 1) * 32 * T::ROW, t * F::TK + s * 32);
            }
            const int turn = v_now;
            v_now = v_next;
            v_next = v_free;
            v_free = turn;
        }
    }
    l = both_sum(l);
    put_row<DT, DP, false>(p, b, g, split, r, qi, head, m, l, o, h);
}

// The splits' results: four channels of a row to a lane.
template <int DT, int DP>
__global__ void __launch_bounds__(256) attend_join(Forward p)
{
    constexpr int ES = elem_size(DT), LANES = DP / 4;
    const int64_t n = (int64_t)p.B * p.Hk * p.rows;
    const int64_t at = ((int64_t)blockIdx.x * 256 + threadIdx.x) / LANES;
    const int d = (int)(((int64_t)blockIdx.x * 256 + threadIdx.x) % LANES) * 4;
    if (at >= n) return;
    const float c = (p.any ? 1.0f : p.scale) * kLog2;
    // eight splits' parts are loaded together
    constexpr int U = 8;
    float m = -__builtin_inff(), l = 0.0f;
    f32x4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int s0 = 0; s0 < p.splits; s0 += U) {
        float from[U], part_l[U];
        f32x4 v[U];
        float to = m;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int64_t i = min(s0 + u, p.splits - 1) * n + at;
            from[u] = p.part_ml[2 * i];
            part_l[u] = p.part_ml[2 * i + 1];
            v[u] = *reinterpret_cast<const f32x4 *>(p.part + i * DP + d);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) to = __builtin_fmaxf(to, from[u]);
        const float by = m == -__builtin_inff() ? 0.0f : exp2_fast((m - to) * c);
        l *= by;
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] *= by;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const float f = s0 + u >= p.splits || from[u] == -__builtin_inff() ? 0.0f : exp2_fast((from[u] - to) * c);
            l = __builtin_fmaf(part_l[u], f, l);
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] = __builtin_fmaf(v[u][i], f, sum[i]);
        }
        m = to;
    }
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    const int64_t problem = at / p.rows;
    const int b = problem / p.Hk, g = problem - (int64_t)b * p.Hk;
    int qi, qj;
    p.row((int)(at - problem * p.rows), qi, qj);
    const int head = g * p.share + qj;
    char *out = p.o + b * p.ob + qi * p.orow + head * p.oh;
    char *rest = p.rest ? p.rest + (((int64_t)b * p.Lq + qi) * p.H + head) * p.D * ES : nullptr;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if (d + i >= p.D) break;
        const float v = sum[i] * inv;
        store_elem<DT>(out, d + i, v);
        if (rest) store_elem<DT>(rest, d + i, v - rounded<DT>(v));
    }
    if (p.stats && d == 0) {
        float *st = p.stats + (((int64_t)b * p.H + head) * p.Lq + qi) * 2;
        st[0] = p.any ? m : m * p.scale;
        st[1] = l == 0.0f ? 0.0f : log2_fast(l) * kLn2;
    }
}

// ---------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------
struct Plan {
    // wq 4: attend_flow, where k and v allow loads to LDS; 5: attend with four wavefronts' rows; 1: with one's
    int wq, tiles, splits, dp;
    bool any;
    bool copies;   // k and v are copied first
};

// A call's shape.  Up to 32 rows: the wavefronts of a workgroup go over the keys in turn, and
// where that leaves fewer than two workgroups a CU the keys are split, for about three of them, at two
// tiles each or more (at one where all tiles together are not more than two a CU).
Plan plan_of(const flashlayer_attention *a)
{
    Plan p{};
    const int64_t rows = (int64_t)a->Lq * (a->Hk ? a->H / a->Hk : 1);
    p.dp = padded_head(a->D);
    const bool flows = !pairs_of(a);
    const int64_t problems = (int64_t)a->B * a->Hk;
    p.wq = rows <= 32 ? 1 : flows ? 4 : 5;
    p.copies = p.wq == 4 && copies_keys(a);
    p.any = p.wq == 1 ? any_of(a) : p.wq == 5;
    const int bq = p.wq == 1 ? 32 : 128, bk = p.wq == 1 ? 128 : 64, bytes = p.dp * elem_size(a->dtype);
    p.tiles = (int)((rows + bq - 1) / bq);
    const int64_t base = problems * p.tiles, keys = (a->Lk + bk - 1) / bk;
    p.splits = 1;
    if (p.wq != 1) {
        p.splits = splits_of(base, keys, p.wq == 4 ? flow_waves(a->dtype, p.dp) : bytes < 384 ? 2 : 1);
    } else if (base > 0 && base < 2 * kCusOfCard) {
        const int64_t want = (3 * kCusOfCard + base - 1) / base;
        p.splits = (int)std::max<int64_t>(1, std::min<int64_t>(want, base * keys <= 2 * kCusOfCard ? keys : keys / 2));
    }
    return p;
}

uint64_t part_bytes(const flashlayer_attention *a, const Plan &p)
{
    const uint64_t rows = (uint64_t)a->B * a->Lq * a->H;
    return align256(size_prod({(uint64_t)p.splits, rows, (uint64_t)p.dp, 4}));
}

uint64_t forward_bytes(const flashlayer_attention *a)
{
    if (!a->B || !a->Lq || !a->H || !a->D) return 0;
    const Plan p = plan_of(a);
    const uint64_t copies = p.copies ? keys_copy_bytes(a) : 0;
    if (p.splits <= 1) return copies;
    return copies + part_bytes(a, p) + align256((uint64_t)p.splits * a->B * a->Lq * a->H * 8);
}

template <int DT, int DP>
int run(Forward &p, const Plan &plan, hipStream_t st)
{
    const void *fn = nullptr;
    size_t lds = 0;
    if (plan.wq == 4 && keys_to_lds(p)) {
        fn = p.words ? (const void *)attend_flow<DT, DP, true> : (const void *)attend_flow<DT, DP, false>;
        lds = Flow<DT, DP>::LDS;
    } else if (plan.wq != 1) {
        fn = (const void *)attend<DT, DP, 4, true>;
        lds = Shape<DT, DP, 4>::LDS;
        p.any = true;
    } else {
        fn = plan.any ? (const void *)attend<DT, DP, 1, true> : (const void *)attend<DT, DP, 1, false>;
        lds = Shape<DT, DP, 1>::LDS;
    }
    if (const int rc = launch_lds(fn, 8ull * p.per_xcd, p, lds, st)) return rc;
    if (p.splits <= 1) return FLASHBEV_OK;
    const uint64_t lanes = (uint64_t)p.B * p.Hk * p.rows * (DP / 4);
    return launch_kernel((const void *)attend_join<DT, DP>, (lanes + 255) / 256, 256, p, 0, st);
}

template <int DT>
int run_width(const flashlayer_attention *a, Forward &p, const Plan &plan, void *workspace, hipStream_t st)
{
    if (plan.copies && a->Lk)
        if (const int rc = copy_keys<DT>(a, p, static_cast<char *>(workspace), st)) return rc;
    switch (plan.dp) {
    case 32: return run<DT, 32>(p, plan, st);
    case 64: return run<DT, 64>(p, plan, st);
    case 96: return run<DT, 96>(p, plan, st);
    default: return run<DT, 128>(p, plan, st);
    }
}

}  // namespace

extern "C" int flashlayer_attention_workspace_size(const flashlayer_attention *args, uint64_t *bytes)
{
    if (!bytes) return FLASHBEV_ERR_NULLPTR;
    if (const int rc = check_attention(args)) return rc;
    *bytes = forward_bytes(args);
    return FLASHBEV_OK;
}

extern "C" int flashlayer_attention_forward(const flashlayer_attention *args, const void *q, const void *k,
                                            const void *v, const void *mask, const int32_t *key_lengths,
                                            void *out, void *rest, float *stats, void *workspace,
                                            uint64_t workspace_bytes, void *stream)
{
    if (const int rc = check_attention(args)) return rc;
    const flashlayer_attention &a = *args;
    const int es = elem_size(a.dtype);
    if (!a.B || !a.Lq || !a.H) return FLASHBEV_OK;
    if (!a.D) return stats ? FLASHBEV_ERR_UNSUPPORTED : FLASHBEV_OK;
    if (!q || !out || (a.Lk && (!k || !v))) return FLASHBEV_ERR_NULLPTR;
    if (a.mask && a.Lk && !mask) return FLASHBEV_ERR_NULLPTR;
    if (!apart(a.B, a.o_batch, a.Lq, a.o_row, a.H, a.o_head, a.D)) return FLASHBEV_ERR_SHAPE;
    const int ms = a.mask == FLASHLAYER_MASK_BOOL ? 1 : a.mask == FLASHLAYER_MASK_ADD_F32 ? 4 : es;
    if (misaligned(q, es) || misaligned(k, es) || misaligned(v, es) || misaligned(out, es) || misaligned(rest, es) ||
        misaligned(stats, 4) || misaligned(key_lengths, 4) || (a.mask && misaligned(mask, ms)))
        return FLASHBEV_ERR_ALIGN;
    const uint64_t need = forward_bytes(args);
    if (const int rc = check_scratch(workspace, workspace_bytes, need)) return rc;
    const uint64_t dense = (uint64_t)a.B * a.Lq * a.H * a.D * es;
    if (const int rc = check_overlaps(
            {{out, span4(a.B, a.o_batch, a.Lq, a.o_row, a.H, a.o_head, a.D, es)},
             {rest, dense},
             {stats, (uint64_t)a.B * a.H * a.Lq * 8},
             {workspace, need}},
            {{q, span4(a.B, a.q_batch, a.Lq, a.q_row, a.H, a.q_head, a.D, es)},
             {k, span4(a.B, a.k_batch, a.Lk, a.k_row, a.Hk, a.k_head, a.D, es)},
             {v, span4(a.B, a.v_batch, a.Lk, a.v_row, a.Hk, a.v_head, a.D, es)},
             {a.mask ? mask : nullptr, span4(a.B, a.mask_batch, a.H, a.mask_head, a.Lq, a.mask_row, a.Lk, ms)},
             {key_lengths, (uint64_t)a.B * 4}}))
        return rc;
    const Plan plan = plan_of(args);
    Forward p{};
    static_cast<Attend &>(p) = attend_of(args);
    p.q = static_cast<const char *>(q);
    p.k = static_cast<const char *>(k);
    p.v = static_cast<const char *>(v);
    p.mask = static_cast<const char *>(mask);
    p.lengths = key_lengths;
    p.o = static_cast<char *>(out);
    p.rest = static_cast<char *>(rest);
    p.stats = stats;
    p.tiles = plan.tiles;
    p.splits = plan.splits;
    p.any = plan.any;
    char *ws = static_cast<char *>(workspace) + (plan.copies ? keys_copy_bytes(args) : 0);
    if (p.splits > 1) {
        p.part = reinterpret_cast<float *>(ws);
        p.part_ml = reinterpret_cast<float *>(ws + part_bytes(args, plan));
    }
    if (const int rc = deal(p, size_prod({(uint64_t)a.B, (uint64_t)a.Hk, (uint64_t)plan.tiles, (uint64_t)plan.splits})))
        return rc;
    const hipStream_t st = static_cast<hipStream_t>(stream);
    if (a.dtype == FLASHBEV_F32) return run_width<FLASHBEV_F32>(args, p, plan, workspace, st);
    return a.dtype == FLASHBEV_F16 ? run_width<FLASHBEV_F16>(args, p, plan, workspace, st) : run_width<FLASHBEV_BF16>(args, p, plan, workspace, st);
}
