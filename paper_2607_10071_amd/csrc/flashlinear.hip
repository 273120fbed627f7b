// The matrix product with bias, activation and residual in its epilogue, and
// its gradients, for AMD MI355X (gfx950).  C ABI: include/block/flashblock.h.
//
// Three products, one kernel.  With an operand's rows over the reduction axis
// ("along") or its columns ("across"),
//
//   forward      out[m,n]  = sum_k x[m,k] W[n,k]     x along,  W along
//   grad_x       gx[m,k]   = sum_n d[m,n] W[n,k]     d along,  W across
//   grad_weight  gw[n,k]   = sum_m d[m,n] x[m,k]     d across, x across
//
// so each is C[i,j] = sum_r A(i,r) B(j,r) with operands in one of two layouts.
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "block_common.h"

namespace {

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x16 __attribute__((ext_vector_type(16)));

// ---------------------------------------------------------------------------
// activations
// ---------------------------------------------------------------------------
constexpr float kSqrtHalf = 0.70710678118654752f;
constexpr float kSqrt2OverPi = 0.79788456080286536f;
constexpr float kInvSqrt2Pi = 0.39894228040143268f;

__device__ __forceinline__ float act_value(int act, float v)
{
    switch (act) {
    case FLASHBLOCK_ACT_RELU: return v > 0.0f ? v : (v == v ? 0.0f : v);
    case FLASHBLOCK_ACT_GELU: return 0.5f * v * (1.0f + erff(v * kSqrtHalf));
    case FLASHBLOCK_ACT_GELU_TANH:
        return 0.5f * v * (1.0f + tanhf(kSqrt2OverPi * (v + 0.044715f * v * v * v)));
    case FLASHBLOCK_ACT_SILU: return v / (1.0f + expf(-v));
    default: return v;
    }
}

__device__ __forceinline__ float act_slope(int act, float v)
{
    switch (act) {
    case FLASHBLOCK_ACT_RELU: return v > 0.0f ? 1.0f : 0.0f;
    case FLASHBLOCK_ACT_GELU:
        return 0.5f * (1.0f + erff(v * kSqrtHalf)) + v * kInvSqrt2Pi * expf(-0.5f * v * v);
    case FLASHBLOCK_ACT_GELU_TANH: {
        const float t = tanhf(kSqrt2OverPi * (v + 0.044715f * v * v * v));
        return 0.5f * (1.0f + t) +
               0.5f * v * (1.0f - t * t) * kSqrt2OverPi * (1.0f + 0.134145f * v * v);
    }
    case FLASHBLOCK_ACT_SILU: {
        const float p = 1.0f / (1.0f + expf(-v));
        return p * (1.0f + v * (1.0f - p));
    }
    default: return 1.0f;
    }
}

// ---------------------------------------------------------------------------
// epilogue: V sums of one row, columns n..n+V-1
// ---------------------------------------------------------------------------
struct Epilogue {
    void *out;
    void *pre;              // null: not wanted
    const void *bias;       // null: none
    const void *residual;   // null: none
    int64_t ldo, ldp, ldr;  // elements
    float scale;
    int act;
    int out_f32;            // out and residual are float32, else the inputs' type
};

template <int DT, int V>
__device__ __forceinline__ void epilogue(const Epilogue &e, int64_t m, int n, int N, float (&v)[V])
{
    const bool whole = n + V <= N;
    const int es = elem_size(DT);
    if (e.bias) {
        if (whole) {
            float b[V];
            load_elems<DT>(static_cast<const char *>(e.bias) + (int64_t)n * es, b);
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] += b[i];
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (n + i < N) v[i] += load_elem<DT>(e.bias, n + i);
        }
    }
    if (e.pre) {
        char *p = static_cast<char *>(e.pre) + (m * e.ldp + n) * es;
        if (whole) {
            store_elems<DT>(p, v);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (n + i < N) store_elem<DT>(p, i, v[i]);
        }
    }
    switch (e.act) {   // the switch outside the loop: one activation's code per call
    case FLASHBLOCK_ACT_RELU:
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = act_value(FLASHBLOCK_ACT_RELU, v[i]);
        break;
    case FLASHBLOCK_ACT_GELU:
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = act_value(FLASHBLOCK_ACT_GELU, v[i]);
        break;
    case FLASHBLOCK_ACT_GELU_TANH:
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = act_value(FLASHBLOCK_ACT_GELU_TANH, v[i]);
        break;
    case FLASHBLOCK_ACT_SILU:
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = act_value(FLASHBLOCK_ACT_SILU, v[i]);
        break;
    default: break;
    }
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] *= e.scale;
    if (e.out_f32) {
        char *p = static_cast<char *>(e.out) + (m * e.ldo + n) * 4;
        const char *r = static_cast<const char *>(e.residual);
        if (r) r += (m * e.ldr + n) * 4;
        if (whole) {
            if (r) {
                float b[V];
                load_elems<FLASHBEV_F32>(r, b);
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] += b[i];
            }
            store_elems<FLASHBEV_F32>(p, v);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (n + i < N)
                    store_elem<FLASHBEV_F32>(p, i, r ? v[i] + load_elem<FLASHBEV_F32>(r, i) : v[i]);
        }
    } else {
        char *p = static_cast<char *>(e.out) + (m * e.ldo + n) * es;
        const char *r = static_cast<const char *>(e.residual);
        if (r) r += (m * e.ldr + n) * es;
        if (whole) {
            if (r) {
                float b[V];
                load_elems<DT>(r, b);
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] += b[i];
            }
            store_elems<DT>(p, v);
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (n + i < N) store_elem<DT>(p, i, r ? v[i] + load_elem<DT>(r, i) : v[i]);
        }
    }
}

// ---------------------------------------------------------------------------
// the tiled product
// ---------------------------------------------------------------------------
// A workgroup computes a BM x BN tile of C in 32 x 32 MFMA blocks, FM x FN of
// them for each of its WM x WN wavefronts, over steps of 128 bytes of the
// reduction axis (64 16-bit or 32 float32 elements).  A granule is 16 bytes: eight
// 16-bit elements, one lane's share of a 32x32x16 MFMA, or four float32, one
// lane's share of four 32x32x2 MFMAs (MFMA q takes element q of both operands'
// granules, so the reduction index runs in the same order on both sides).
//
// LDS layout.  Along: row i holds its 8 granules, granule g at place g ^ (i & 7),
// so that 8 lanes reading the same granule of 8 rows hit 8 different 16-byte
// places.  Across: row r of the reduction axis holds the tile's columns.  16-bit
// columns are read transposed (ds_read_b64_tr_b16: 16 lanes take a 4 x 16 block
// and each ends with one column's 4 rows); the 32-byte column blocks of row r
// stand at places XORed with (r & 3) + 4 (r >> 3 & 1), so that the 8 rows that one
// instruction touches use different banks.  float32 columns are read as
// they stand.
struct Gemm {
    const char *a, *b;
    int64_t lda, ldb;          // bytes
    int rows, cols;            // of C
    int red;                   // length of the reduction axis
    int tiles_m, tiles_n;
    int split;                 // workgroups that share a tile's reduction axis
    int steps;                 // reduction steps for each of them
    float *partial;            // split > 1: [split][rows][pld] float32 sums
    int64_t pld;
    Epilogue e;
};

template <int DT>
__device__ __forceinline__ void mma(f32x16 &c, const u32x4 &a, const u32x4 &b)
{
    if constexpr (DT == FLASHBEV_BF16) {
        c = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a),
                                                    __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
    } else if constexpr (DT == FLASHBEV_F16) {
        c = __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(f16x8, a),
                                                   __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    } else {
        const f32x4 fa = __builtin_bit_cast(f32x4, a), fb = __builtin_bit_cast(f32x4, b);
#pragma unroll
        for (int q = 0; q < 4; ++q)
            c = __builtin_amdgcn_mfma_f32_32x32x2f32(fa[q], fb[q], c, 0, 0, 0);
    }
}

// 16 bytes at element `i` of a row that ends at element `end`; zeros past it
template <int DT>
__device__ __forceinline__ u32x4 load_granule_edge(const char *row, int i, int end)
{
    constexpr int E = 16 / elem_size(DT);
    u32x4 v = {0, 0, 0, 0};
    if (i + E <= end) {
        v = load16(row + (int64_t)i * elem_size(DT));
    } else {
#pragma unroll
        for (int q = 0; q < E; ++q) {
            if (i + q >= end) continue;
            if constexpr (DT == FLASHBEV_F32) {
                v[q] = reinterpret_cast<const uint32_t *>(row)[i + q];
            } else {
                v[q >> 1] |= (uint32_t)reinterpret_cast<const uint16_t *>(row)[i + q]
                             << (16 * (q & 1));
            }
        }
    }
    return v;
}

// One operand's tile of R rows (or columns) of C on its way from memory to LDS.
template <int DT, bool ACROSS, int R, int NT>
struct Tile {
    static constexpr int ES = elem_size(DT);
    static constexpr int E = 16 / ES;
    static constexpr int KT = 128 / ES;        // reduction elements per step
    static constexpr int BYTES = R * 128;
    static constexpr int G = R * 8 / NT;       // granules per thread
    static constexpr int GPR = ACROSS ? R * ES / 16 : 8;   // granules per LDS row
    static constexpr int PAIRS = R / 16;       // 32-byte column blocks (16-bit, across)
    static_assert(R * 8 % NT == 0, "whole granules per thread");

    // the step's granules, `left` reduction elements from it on (rows of C past
    // the last one repeat it: their sums are not stored)
    template <bool EDGE>
    static __device__ __forceinline__ void load(u32x4 (&v)[G], const char *base, int64_t ld, int c0,
                                                int cend, int r0, int rend, int tid)
    {
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const int q = tid + i * NT;
            const int row = q / GPR, g = q % GPR;
            if constexpr (!ACROSS) {
                const int c = min(c0 + row, cend - 1);
                const char *p = base + (int64_t)c * ld;
                if constexpr (EDGE)
                    v[i] = load_granule_edge<DT>(p, r0 + g * E, rend);
                else
                    v[i] = load16(p + (int64_t)(r0 + g * E) * ES);
            } else {
                const char *p = base + (int64_t)(r0 + row) * ld;
                if constexpr (EDGE) {
                    if (r0 + row < rend)
                        v[i] = load_granule_edge<DT>(p, c0 + g * E, cend);
                    else
                        v[i] = u32x4{0, 0, 0, 0};
                } else {
                    v[i] = load16(p + (int64_t)(c0 + g * E) * ES);
                }
            }
        }
    }

    static __device__ __forceinline__ int swizzle(int r)
    {
        return ((r & 3) | ((r >> 3 & 1) << 2)) & (PAIRS - 1);
    }

    static __device__ __forceinline__ void store(const u32x4 (&v)[G], char *lds, int tid)
    {
#pragma unroll
        for (int i = 0; i < G; ++i) {
            const int q = tid + i * NT;
            const int row = q / GPR, g = q % GPR;
            int place = g;
            if constexpr (!ACROSS) place = g ^ (row & 7);
            else if constexpr (ES == 2) place = g ^ (swizzle(row) << 1);
            *reinterpret_cast<u32x4 *>(lds + (row * GPR + place) * 16) = v[i];
        }
    }

    // the lane's granule g of reduction elements for column (row of C) c0 + lane % 32
    static __device__ __forceinline__ u32x4 fragment(const char *lds, int c0, int kk, int lane)
    {
        const int h = lane >> 5;
        if constexpr (!ACROSS) {
            const int row = c0 + (lane & 31), g = 2 * kk + h;
            return *reinterpret_cast<const u32x4 *>(lds + (row * 8 + (g ^ (row & 7))) * 16);
        } else if constexpr (ES == 2) {
            const int j = lane & 15;
            const int pair = (c0 >> 4) + (lane >> 4 & 1);
            const int r = kk * 16 + h * 8 + (j >> 2);
            u32x4 v;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int rr = r + 4 * q;
                const char *p = lds + rr * (R * 2) + ((pair ^ swizzle(rr)) * 32) + (j & 3) * 8;
                const s16x4 t = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
                    (__attribute__((address_space(3))) s16x4 *)(p));
                const uint64_t w = __builtin_bit_cast(uint64_t, t);
                v[2 * q] = (uint32_t)w;
                v[2 * q + 1] = (uint32_t)(w >> 32);
            }
            return v;
        } else {
            const int r = (2 * kk + h) * 4;
            u32x4 v;
#pragma unroll
            for (int q = 0; q < 4; ++q)
                v[q] = *reinterpret_cast<const uint32_t *>(lds + ((r + q) * R + c0 + (lane & 31)) * 4);
            return v;
        }
    }
};

template <int DT, bool AX, bool BX, int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__(WM *WN * 64) linear_tiles(Gemm p)
{
    constexpr int NT = WM * WN * 64;
    constexpr int TM = BM / WM, TN = BN / WN;      // a wavefront's part of the tile
    constexpr int FM = TM / 32, FN = TN / 32;
    using TA = Tile<DT, AX, BM, NT>;
    using TB = Tile<DT, BX, BN, NT>;
    constexpr int KT = TA::KT;
    constexpr int STAGE = TA::BYTES + TB::BYTES;
    constexpr int ESTRIDE = TN + 4;                // floats; epilogue rows, 16-byte aligned
    constexpr int EBYTES = WM * WN * 32 * ESTRIDE * 4;
    __shared__ __attribute__((aligned(16))) char lds[2 * STAGE > EBYTES ? 2 * STAGE : EBYTES];

    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int wm = wave / WN, wn = wave % WN;
    const int tile = blockIdx.x / p.split, part = blockIdx.x % p.split;
    const int m0 = tile / p.tiles_n * BM, n0 = tile % p.tiles_n * BN;

    f32x16 acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;

    const int total = (p.red + KT - 1) / KT;
    const int s0 = part * p.steps, s1 = min(total, s0 + p.steps);
    // tiles that hang over an "across" operand's columns, and the last step of an
    // axis that is no multiple of a step, take the checked loads
    const bool edge = (AX && m0 + BM > p.rows) || (BX && n0 + BN > p.cols);
    u32x4 va[TA::G], vb[TB::G];
    auto fetch = [&](int s) {
        if (edge || (s + 1) * KT > p.red) {
            TA::template load<true>(va, p.a, p.lda, m0, p.rows, s * KT, p.red, tid);
            TB::template load<true>(vb, p.b, p.ldb, n0, p.cols, s * KT, p.red, tid);
        } else {
            TA::template load<false>(va, p.a, p.lda, m0, p.rows, s * KT, p.red, tid);
            TB::template load<false>(vb, p.b, p.ldb, n0, p.cols, s * KT, p.red, tid);
        }
    };
    if (s0 < s1) fetch(s0);
    for (int s = s0; s < s1; ++s) {
        char *la = lds + (s - s0 & 1) * STAGE, *lb = la + TA::BYTES;
        TA::store(va, la, tid);
        TB::store(vb, lb, tid);
        __syncthreads();
        if (s + 1 < s1) fetch(s + 1);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
            u32x4 fa[FM], fb[FN];
#pragma unroll
            for (int i = 0; i < FM; ++i) fa[i] = TA::fragment(la, wm * TM + i * 32, kk, lane);
#pragma unroll
            for (int j = 0; j < FN; ++j) fb[j] = TB::fragment(lb, wn * TN + j * 32, kk, lane);
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) mma<DT>(acc[i][j], fa[i], fb[j]);
        }
    }
    __syncthreads();

    // Epilogue: the MFMA leaves a lane with one column's 16 rows; through LDS,
    // 32 rows at a time, each lane gets a row's consecutive columns, so that
    // bias, residual and output move in 16-byte vectors.
    float *stage = reinterpret_cast<float *>(lds) + wave * 32 * ESTRIDE;
#pragma unroll
    for (int i = 0; i < FM; ++i) {
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int e = 0; e < 16; ++e)
                stage[(8 * (e / 4) + 4 * (lane >> 5) + e % 4) * ESTRIDE + j * 32 + (lane & 31)] =
                    acc[i][j][e];
        wave_lds_sync();
        constexpr int V = 16 / elem_size(DT);
        constexpr int LPR = TN / V, RPP = 64 / LPR;    // lanes per row, rows per pass
#pragma unroll
        for (int q = 0; q < 32 / RPP; ++q) {
            const int r = q * RPP + lane / LPR, c = lane % LPR * V;
            const int m = m0 + wm * TM + i * 32 + r, n = n0 + wn * TN + c;
            float v[V];
#pragma unroll
            for (int e = 0; e < V; e += 4) {
                const f32x4 w = *reinterpret_cast<const f32x4 *>(stage + r * ESTRIDE + c + e);
#pragma unroll
                for (int k = 0; k < 4; ++k) v[e + k] = w[k];
            }
            if (m >= p.rows || n >= p.cols) continue;
            if (p.split > 1)
                store_elems<FLASHBEV_F32>(p.partial + ((int64_t)part * p.rows + m) * p.pld + n, v);
            else
                epilogue<DT>(p.e, m, n, p.cols, v);
        }
        wave_lds_sync();
    }
}

// ---------------------------------------------------------------------------
// sums of the parts of a split reduction axis, in their order
// ---------------------------------------------------------------------------
struct Join {
    const float *partial;   // [split][rows][pld], pld a multiple of 8
    int64_t pld;
    int rows, cols, split;
    Epilogue e;
};

template <int DT>
__global__ void __launch_bounds__(256) linear_join(Join p)
{
    constexpr int V = 16 / elem_size(DT);
    const int per_row = (p.cols + V - 1) / V;
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t m = i / per_row;
    if (m >= p.rows) return;
    const int n = (int)(i % per_row) * V;
    float v[V];
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = 0.0f;
    const float *src = p.partial + m * p.pld + n;
    for (int s = 0; s < p.split; ++s) {
        float w[V];
        load_elems<FLASHBEV_F32>(src + (int64_t)s * p.rows * p.pld, w);
#pragma unroll
        for (int e = 0; e < V; ++e) v[e] += w[e];
    }
    epilogue<DT>(p.e, m, n, p.cols, v);
}

// ---------------------------------------------------------------------------
// d = scale act'(pre) grad_out in the inputs' type, and its column sums
// ---------------------------------------------------------------------------
// A workgroup takes 256 columns of a range of rows; 32 lanes share a row, 8
// columns each, and 8 rows are in flight.  Its column sums (float32, of the
// unrounded values) go to its range's row of `partial`; column_join adds those in
// order.
struct Slope {
    const void *grad;       // [M, N], DT or float32
    const void *pre;        // null without an activation
    void *d;                // null: column sums alone
    float *partial;         // [ranges][pld], null: no column sums
    int64_t ldg, ldp, ldd, pld;   // elements
    int M, N, rows;         // rows of a range
    int col_blocks;
    int act, grad_f32;
    float scale;
};

template <int DT>
__global__ void __launch_bounds__(256) linear_slope(Slope p)
{
    const int cb = blockIdx.x % p.col_blocks, range = blockIdx.x / p.col_blocks;
    const int n = cb * 256 + (threadIdx.x & 31) * 8;
    const int64_t r0 = (int64_t)range * p.rows, r1 = min((int64_t)p.M, r0 + p.rows);
    constexpr int es = elem_size(DT);
    float sum[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] = 0.0f;
    if (n < p.N) {
        const bool whole = n + 8 <= p.N;
        for (int64_t m = r0 + (threadIdx.x >> 5); m < r1; m += 8) {
            float g[8], v[8];
            const char *gp = static_cast<const char *>(p.grad) + (m * p.ldg + n) * (p.grad_f32 ? 4 : es);
            const char *vp = static_cast<const char *>(p.pre) + (m * p.ldp + n) * es;
            if (whole) {
                if (p.grad_f32) load_elems<FLASHBEV_F32>(gp, g);
                else load_elems<DT>(gp, g);
                if (p.act) load_elems<DT>(vp, v);
            } else {
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const bool in = n + e < p.N;
                    g[e] = !in ? 0.0f : p.grad_f32 ? load_elem<FLASHBEV_F32>(gp, e) : load_elem<DT>(gp, e);
                    v[e] = in && p.act ? load_elem<DT>(vp, e) : 0.0f;
                }
            }
            if (p.act) {
#pragma unroll
                for (int e = 0; e < 8; ++e) g[e] *= act_slope(p.act, v[e]);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                g[e] *= p.scale;
                sum[e] += g[e];
            }
            if (p.d) {
                char *dp = static_cast<char *>(p.d) + (m * p.ldd + n) * es;
                if (whole) {
                    store_elems<DT>(dp, g);
                } else {
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        if (n + e < p.N) store_elem<DT>(dp, e, g[e]);
                }
            }
        }
    }
    if (!p.partial) return;
    __shared__ float part[8][256 + 8];
#pragma unroll
    for (int e = 0; e < 8; ++e) part[threadIdx.x >> 5][(threadIdx.x & 31) * 8 + e] = sum[e];
    __syncthreads();
    const int c = cb * 256 + threadIdx.x;
    float s = 0.0f;
#pragma unroll
    for (int r = 0; r < 8; ++r) s += part[r][threadIdx.x];
    if (c < p.N) p.partial[(int64_t)range * p.pld + c] = s;
}

// out[n] = sum over ranges of partial[range][n], in `DT`; 16 columns per workgroup
struct ColumnJoin {
    const float *partial;
    int64_t pld;
    int ranges, N;
    void *out;
};

template <int DT>
__global__ void __launch_bounds__(256) column_join(ColumnJoin p)
{
    const int n = blockIdx.x * 16 + (threadIdx.x & 15), r0 = threadIdx.x >> 4;
    float s = 0.0f;
    if (n < p.N)
        for (int r = r0; r < p.ranges; r += 16) s += p.partial[(int64_t)r * p.pld + n];
    __shared__ float part[16][17];
    part[r0][threadIdx.x & 15] = s;
    __syncthreads();
    if (r0 != 0 || n >= p.N) return;
    s = 0.0f;
#pragma unroll
    for (int r = 0; r < 16; ++r) s += part[r][threadIdx.x];
    store_elem<DT>(p.out, n, s);
}

// ---------------------------------------------------------------------------
// host: plans and launches
// ---------------------------------------------------------------------------
constexpr int kCus = 256;

uint64_t round_up(uint64_t v, uint64_t to) { return (v + to - 1) / to * to; }

struct TilePlan {
    int bm, bn, split, steps;
    uint64_t workspace;    // bytes of partial sums
};

TilePlan plan_tiles(int64_t rows, int64_t cols, int64_t red, int dt)
{
    TilePlan t;
    const int kt = 128 / elem_size(dt);
    const int64_t total = (red + kt - 1) / kt;
    t.bm = t.bn = 128;
    int64_t tiles = ((rows + 127) / 128) * ((cols + 127) / 128);
    if (tiles < kCus) {
        t.bm = t.bn = 64;
        tiles = ((rows + 63) / 64) * ((cols + 63) / 64);
    }
    // split the reduction axis until the chip has two workgroups per CU, in
    // parts of four steps or more
    int64_t split = tiles > 0 ? 2 * kCus / tiles : 1;
    if (split > total / 4) split = total / 4;
    if (split < 1) split = 1;
    t.steps = (int)((total + split - 1) / split);
    if (t.steps < 1) t.steps = 1;
    split = (total + t.steps - 1) / t.steps;
    t.split = (int)(split < 1 ? 1 : split);
    t.workspace = t.split > 1 ? round_up((uint64_t)t.split * rows * round_up(cols, 8) * 4, 256) : 0;
    return t;
}

template <int DT, bool AX, bool BX>
int launch_tiles(Gemm &g, const TilePlan &t, hipStream_t st)
{
    const uint64_t blocks = (uint64_t)g.tiles_m * g.tiles_n * g.split;
    if (t.bm == 128)
        return launch_kernel((const void *)linear_tiles<DT, AX, BX, 128, 128, 2, 2>, blocks, 256, g,
                             0, st);
    return launch_kernel((const void *)linear_tiles<DT, AX, BX, 64, 64, 2, 2>, blocks, 256, g, 0, st);
}

// C = A B^T through the epilogue; `workspace` of plan_tiles(...).workspace bytes
template <bool AX, bool BX>
int product(int dt, const void *a, int64_t lda, const void *b, int64_t ldb, int64_t rows,
            int64_t cols, int64_t red, const Epilogue &e, void *workspace, hipStream_t st)
{
    if (rows == 0 || cols == 0) return FLASHBEV_OK;
    const TilePlan t = plan_tiles(rows, cols, red, dt);
    const int es = elem_size(dt);
    Gemm g{};
    g.a = static_cast<const char *>(a);
    g.b = static_cast<const char *>(b);
    g.lda = lda * es;
    g.ldb = ldb * es;
    g.rows = (int)rows;
    g.cols = (int)cols;
    g.red = (int)red;
    g.tiles_m = (int)((rows + t.bm - 1) / t.bm);
    g.tiles_n = (int)((cols + t.bn - 1) / t.bn);
    g.split = t.split;
    g.steps = t.steps;
    g.partial = static_cast<float *>(workspace);
    g.pld = (int64_t)round_up(cols, 8);
    g.e = e;
    int rc = dt == FLASHBEV_F32   ? launch_tiles<FLASHBEV_F32, AX, BX>(g, t, st)
             : dt == FLASHBEV_F16 ? launch_tiles<FLASHBEV_F16, AX, BX>(g, t, st)
                                  : launch_tiles<FLASHBEV_BF16, AX, BX>(g, t, st);
    if (rc || t.split == 1) return rc;
    Join j{g.partial, g.pld, g.rows, g.cols, t.split, e};
    const uint64_t vecs = (uint64_t)rows * ((cols + 16 / es - 1) / (16 / es));
    const void *fn = dt == FLASHBEV_F32   ? (const void *)linear_join<FLASHBEV_F32>
                     : dt == FLASHBEV_F16 ? (const void *)linear_join<FLASHBEV_F16>
                                          : (const void *)linear_join<FLASHBEV_BF16>;
    return launch_kernel(fn, (vecs + 255) / 256, 256, j, 0, st);
}

int check_sizes(const flashblock_linear *p)
{
    if (!p) return FLASHBEV_ERR_NULLPTR;
    if (p->M < 0 || p->K < 0 || p->N < 0) return FLASHBEV_ERR_SHAPE;
    if (!known_dtype(p->dtype) || (p->out_dtype != p->dtype && p->out_dtype != FLASHBEV_F32))
        return FLASHBEV_ERR_DTYPE;
    if (p->act < FLASHBLOCK_ACT_NONE || p->act > FLASHBLOCK_ACT_SILU || !finite_value(p->scale))
        return FLASHBEV_ERR_VALUE;
    if (p->M > 0x7fffffff || p->K > FLASHBLOCK_WIDTH_MAX || p->N > FLASHBLOCK_WIDTH_MAX)
        return FLASHBEV_ERR_UNSUPPORTED;
    return FLASHBEV_OK;
}

// a tensor of `rows` rows: its stride and pointer
int check_rows(const void *p, int64_t rows, int64_t ld, int64_t width, int es)
{
    if (rows == 0 || width == 0) return FLASHBEV_OK;
    if (!p) return FLASHBEV_ERR_NULLPTR;
    if (ld < width) return FLASHBEV_ERR_SHAPE;
    if (ld > FLASHBLOCK_LD_MAX) return FLASHBEV_ERR_UNSUPPORTED;
    return misaligned(p, es) ? FLASHBEV_ERR_ALIGN : FLASHBEV_OK;
}

int check_workspace(const void *ws, uint64_t have, uint64_t need)
{
    if (need == 0) return FLASHBEV_OK;
    if (!ws) return FLASHBEV_ERR_NULLPTR;
    if (misaligned(ws, 256)) return FLASHBEV_ERR_ALIGN;
    return have < need ? FLASHBEV_ERR_SCRATCH : FLASHBEV_OK;
}

struct Range {
    const void *p;
    uint64_t n;
};

// The backward's workspace: d, then the column sums, then the products' partial
// sums (grad_weight's, and after it grad_x's in the same place).
struct BackwardPlan {
    bool slope;            // d is a tensor of its own
    bool column_sums;
    int ranges, range_rows;
    int64_t ldd;
    uint64_t d_bytes, sum_bytes, partial_bytes, total;
};

BackwardPlan plan_backward(const flashblock_linear *p, bool want_x, bool want_w, bool want_b)
{
    BackwardPlan b{};
    const int es = elem_size(p->dtype);
    b.slope = (want_x || want_w) && (p->act != FLASHBLOCK_ACT_NONE || p->out_dtype != p->dtype);
    b.column_sums = want_b;
    b.ldd = (int64_t)round_up((uint64_t)p->N, 8);
    b.d_bytes = b.slope ? round_up((uint64_t)p->M * b.ldd * es, 256) : 0;
    // ranges: about four workgroups per CU, of 32 rows or more
    const int64_t col_blocks = (p->N + 255) / 256;
    int64_t ranges = col_blocks > 0 ? 4 * kCus / col_blocks : 1;
    if (ranges > 256) ranges = 256;
    if (ranges > p->M / 32) ranges = p->M / 32;
    if (ranges < 1) ranges = 1;
    b.range_rows = (int)((p->M + ranges - 1) / ranges);
    if (b.range_rows < 1) b.range_rows = 1;
    b.ranges = (int)((p->M + b.range_rows - 1) / b.range_rows);
    if (b.ranges < 1) b.ranges = 1;
    b.sum_bytes = want_b ? round_up((uint64_t)b.ranges * b.ldd * 4, 256) : 0;
    if (want_w) b.partial_bytes = plan_tiles(p->N, p->K, p->M, p->dtype).workspace;
    if (want_x) {
        const uint64_t w = plan_tiles(p->M, p->K, p->N, p->dtype).workspace;
        if (w > b.partial_bytes) b.partial_bytes = w;
    }
    b.total = b.d_bytes + b.sum_bytes + b.partial_bytes;
    return b;
}

}  // namespace

extern "C" {

int flashblock_linear_workspace_size(const flashblock_linear *p, uint64_t *bytes)
{
    if (!bytes) return FLASHBEV_ERR_NULLPTR;
    if (const int rc = check_sizes(p)) return rc;
    *bytes = plan_tiles(p->M, p->N, p->K, p->dtype).workspace;
    return FLASHBEV_OK;
}

int flashblock_linear_forward(const flashblock_linear *p, const void *x, const void *weight,
                              const void *bias, const void *residual, void *out, void *pre,
                              void *workspace, uint64_t workspace_bytes, void *stream)
{
    int rc = check_sizes(p);
    if (rc) return rc;
    const int es = elem_size(p->dtype), os = elem_size(p->out_dtype);
    if (p->M == 0 || p->N == 0) return FLASHBEV_OK;
    if ((rc = check_rows(x, p->M, p->ldx, p->K, es)) ||
        (rc = check_rows(weight, p->N, p->ldw, p->K, es)) ||
        (rc = check_rows(out, p->M, p->ldo, p->N, os)))
        return rc;
    if (residual && (rc = check_rows(residual, p->M, p->ldr, p->N, os))) return rc;
    if (pre && (rc = check_rows(pre, p->M, p->ldp, p->N, es))) return rc;
    if (misaligned(bias, es)) return FLASHBEV_ERR_ALIGN;
    const uint64_t need = plan_tiles(p->M, p->N, p->K, p->dtype).workspace;
    if ((rc = check_workspace(workspace, workspace_bytes, need))) return rc;
    const bool in_place = residual == out && p->ldr == p->ldo;
    const Range ins[] = {{x, span_bytes(p->M, p->ldx, p->K, es)},
                         {weight, span_bytes(p->N, p->ldw, p->K, es)},
                         {bias, (uint64_t)p->N * es},
                         {residual, span_bytes(p->M, p->ldr, p->N, os)}};
    const Range outs[] = {{out, span_bytes(p->M, p->ldo, p->N, os)},
                          {pre, span_bytes(p->M, p->ldp, p->N, es)},
                          {workspace, need}};
    for (int o = 0; o < 3; ++o) {
        for (int i = 0; i < 4; ++i)
            if (!(o == 0 && i == 3 && in_place) &&
                ranges_overlap(outs[o].p, outs[o].n, ins[i].p, ins[i].n))
                return FLASHBEV_ERR_ALIAS;
        for (int q = 0; q < o; ++q)
            if (ranges_overlap(outs[o].p, outs[o].n, outs[q].p, outs[q].n)) return FLASHBEV_ERR_ALIAS;
    }
    Epilogue e{out, pre, bias, residual, p->ldo, p->ldp, p->ldr, p->scale, p->act,
               p->out_dtype == FLASHBEV_F32};
    return product<false, false>(p->dtype, x, p->ldx, weight, p->ldw, p->M, p->N, p->K, e, workspace,
                                 static_cast<hipStream_t>(stream));
}

int flashblock_linear_backward_workspace_size(const flashblock_linear *p, int32_t want_x,
                                              int32_t want_weight, int32_t want_bias,
                                              uint64_t *bytes)
{
    if (!bytes) return FLASHBEV_ERR_NULLPTR;
    if (const int rc = check_sizes(p)) return rc;
    *bytes = plan_backward(p, want_x, want_weight, want_bias).total;
    return FLASHBEV_OK;
}

int flashblock_linear_backward(const flashblock_linear *p, const void *grad_out, const void *x,
                               const void *weight, const void *pre, void *grad_x, int64_t ldgx,
                               void *grad_weight, int64_t ldgw, void *grad_bias, void *workspace,
                               uint64_t workspace_bytes, void *stream)
{
    int rc = check_sizes(p);
    if (rc) return rc;
    const int es = elem_size(p->dtype), os = elem_size(p->out_dtype);
    // gradients without elements have no address and nothing to write
    const bool has_x = p->M > 0 && p->K > 0, has_w = p->N > 0 && p->K > 0, has_b = p->N > 0;
    if (!grad_x && !grad_weight && !grad_bias && has_x && has_w && has_b)
        return FLASHBEV_ERR_NULLPTR;
    const bool want_x = grad_x && has_x, want_w = grad_weight && has_w, want_b = grad_bias && has_b;
    if (!want_x && !want_w && !want_b) return FLASHBEV_OK;
    if ((rc = check_rows(grad_out, p->M, p->ldo, p->N, os))) return rc;
    if (want_w && (rc = check_rows(x, p->M, p->ldx, p->K, es))) return rc;
    if (want_x && (rc = check_rows(weight, p->N, p->ldw, p->K, es))) return rc;
    if (p->act != FLASHBLOCK_ACT_NONE && (rc = check_rows(pre, p->M, p->ldp, p->N, es))) return rc;
    if (want_x && (rc = check_rows(grad_x, p->M, ldgx, p->K, es))) return rc;
    if (want_w && (rc = check_rows(grad_weight, p->N, ldgw, p->K, es))) return rc;
    if (misaligned(grad_bias, es)) return FLASHBEV_ERR_ALIGN;
    const BackwardPlan b = plan_backward(p, want_x, want_w, want_b);
    if ((rc = check_workspace(workspace, workspace_bytes, b.total))) return rc;
    const Range ins[] = {
        {grad_out, span_bytes(p->M, p->ldo, p->N, os)},
        {want_w ? x : nullptr, span_bytes(p->M, p->ldx, p->K, es)},
        {want_x ? weight : nullptr, span_bytes(p->N, p->ldw, p->K, es)},
        {p->act != FLASHBLOCK_ACT_NONE ? pre : nullptr, span_bytes(p->M, p->ldp, p->N, es)}};
    const Range outs[] = {{want_x ? grad_x : nullptr, span_bytes(p->M, ldgx, p->K, es)},
                          {want_w ? grad_weight : nullptr, span_bytes(p->N, ldgw, p->K, es)},
                          {want_b ? grad_bias : nullptr, (uint64_t)p->N * es},
                          {workspace, b.total}};
    for (int o = 0; o < 4; ++o) {
        for (int i = 0; i < 4; ++i)
            if (ranges_overlap(outs[o].p, outs[o].n, ins[i].p, ins[i].n)) return FLASHBEV_ERR_ALIAS;
        for (int q = 0; q < o; ++q)
            if (ranges_overlap(outs[o].p, outs[o].n, outs[q].p, outs[q].n)) return FLASHBEV_ERR_ALIAS;
    }
    hipStream_t st = static_cast<hipStream_t>(stream);
    char *ws = static_cast<char *>(workspace);
    const int dt = p->dtype;
    const void *d = grad_out;
    int64_t ldd = p->ldo;
    float alpha = p->scale;
    if (b.slope || b.column_sums) {
        Slope s{};
        s.grad = grad_out;
        s.pre = pre;
        s.ldg = p->ldo;
        s.ldp = p->ldp;
        s.ldd = b.ldd;
        s.pld = b.ldd;
        s.M = (int)p->M;
        s.N = p->N;
        s.rows = b.range_rows;
        s.col_blocks = (p->N + 255) / 256;
        s.act = p->act;
        s.grad_f32 = p->out_dtype == FLASHBEV_F32;
        s.scale = p->scale;
        s.d = b.slope ? ws : nullptr;
        s.partial = b.column_sums ? reinterpret_cast<float *>(ws + b.d_bytes) : nullptr;
        const void *fn = dt == FLASHBEV_F32   ? (const void *)linear_slope<FLASHBEV_F32>
                         : dt == FLASHBEV_F16 ? (const void *)linear_slope<FLASHBEV_F16>
                                              : (const void *)linear_slope<FLASHBEV_BF16>;
        if ((rc = launch_kernel(fn, (uint64_t)s.col_blocks * b.ranges, 256, s, 0, st))) return rc;
        if (b.slope) {
            d = ws;
            ldd = b.ldd;
            alpha = 1.0f;
        }
        if (b.column_sums) {
            ColumnJoin c{s.partial, b.ldd, b.ranges, p->N, grad_bias};
            fn = dt == FLASHBEV_F32   ? (const void *)column_join<FLASHBEV_F32>
                 : dt == FLASHBEV_F16 ? (const void *)column_join<FLASHBEV_F16>
                                      : (const void *)column_join<FLASHBEV_BF16>;
            if ((rc = launch_kernel(fn, (uint64_t)(p->N + 15) / 16, 256, c, 0, st))) return rc;
        }
    }
    void *partial = ws + b.d_bytes + b.sum_bytes;
    if (want_w) {
        Epilogue e{grad_weight, nullptr, nullptr, nullptr, ldgw, 0, 0, alpha, FLASHBLOCK_ACT_NONE,
                   dt == FLASHBEV_F32};
        if ((rc = product<true, true>(dt, d, ldd, x, p->ldx, p->N, p->K, p->M, e, partial, st)))
            return rc;
    }
    if (want_x) {
        Epilogue e{grad_x, nullptr, nullptr, nullptr, ldgx, 0, 0, alpha, FLASHBLOCK_ACT_NONE,
                   dt == FLASHBEV_F32};
        if ((rc = product<false, true>(dt, d, ldd, weight, p->ldw, p->M, p->K, p->N, e, partial, st)))
            return rc;
    }
    return FLASHBEV_OK;
}

}  // extern "C"
